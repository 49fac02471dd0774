// Instances of the grouped product: X W_e^T in 8-bit integers.
#include "lgn_grouped.cuh"

namespace lgn {

GmKernels gm_int8_kernels() {
    static const GmKernel table[] = {
        gm_kernel<kGmInt8, 256, 2, kGmRows, true, LGN_BF16>(4.0f, 0.30f, 1.5f), gm_kernel<kGmInt8, 256, 2, kGmRows, true, LGN_F32>(4.0f, 0.30f, 2.5f),
        gm_kernel<kGmInt8, 128, 2, kGmRows, true, LGN_BF16>(3.8f, 0.2f, 1.0f), gm_kernel<kGmInt8, 128, 2, kGmRows, true, LGN_F32>(3.8f, 0.2f, 1.5f),
        gm_kernel<kGmInt8, 128, 1, kGmRows, true, LGN_BF16>(3.5f, 0.25f, 1.0f), gm_kernel<kGmInt8, 128, 1, kGmRows, true, LGN_F32>(3.5f, 0.25f, 1.5f),
        gm_kernel<kGmInt8, 32, 1, kGmSwap, true, LGN_BF16>(3.5f, 0.45f, 0.5f), gm_kernel<kGmInt8, 32, 1, kGmSwap, true, LGN_F32>(3.5f, 0.45f, 0.5f),
        gm_kernel<kGmInt8, 64, 1, kGmSwap, true, LGN_BF16>(3.5f, 0.5f, 0.6f), gm_kernel<kGmInt8, 64, 1, kGmSwap, true, LGN_F32>(3.5f, 0.5f, 0.6f)};
    return {table, (int)(sizeof table / sizeof table[0])};
}

}  // namespace lgn
