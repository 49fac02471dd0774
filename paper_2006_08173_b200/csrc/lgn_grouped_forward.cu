// Instances of the grouped product: X W_e^T in bf16.
#include "lgn_grouped.cuh"

namespace lgn {

GmKernels gm_forward_kernels() {
    static const GmKernel table[] = {
        gm_kernel<kGmBf16, 256, 2, kGmRows, true, LGN_BF16>(4.0f, 0.30f, 1.5f), gm_kernel<kGmBf16, 256, 2, kGmRows, true, LGN_F32>(4.0f, 0.30f, 2.5f),
        gm_kernel<kGmBf16, 256, 1, kGmRows, true, LGN_BF16>(3.8f, 0.36f, 1.6f), gm_kernel<kGmBf16, 256, 1, kGmRows, true, LGN_F32>(3.8f, 0.36f, 2.2f),
        gm_kernel<kGmBf16, 128, 1, kGmRows, true, LGN_BF16>(3.5f, 0.25f, 1.0f), gm_kernel<kGmBf16, 128, 1, kGmRows, true, LGN_F32>(3.5f, 0.25f, 1.5f),
        gm_kernel<kGmBf16, 32, 1, kGmSwap, true, LGN_BF16>(3.5f, 0.45f, 0.5f), gm_kernel<kGmBf16, 32, 1, kGmSwap, true, LGN_F32>(3.5f, 0.45f, 0.5f),
        gm_kernel<kGmBf16, 64, 1, kGmSwap, true, LGN_BF16>(3.5f, 0.5f, 0.6f), gm_kernel<kGmBf16, 64, 1, kGmSwap, true, LGN_F32>(3.5f, 0.5f, 0.6f)};
    return {table, (int)(sizeof table / sizeof table[0])};
}

}  // namespace lgn
