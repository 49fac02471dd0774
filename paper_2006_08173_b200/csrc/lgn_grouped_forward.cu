// Instances of the grouped product: X W_e^T in bf16.
#include "lgn_grouped.cuh"

namespace lgn {

GmKernels gm_forward_kernels() {
    static const GmKernel table[] = {
        gm_kernel<kGmBf16, 256, 2, kGmTurn, true, LGN_BF16>(), gm_kernel<kGmBf16, 256, 2, kGmTurn, true, LGN_F32>(),
        gm_kernel<kGmBf16, 256, 2, kGmRows, true, LGN_BF16>(), gm_kernel<kGmBf16, 256, 2, kGmRows, true, LGN_F32>(),
        gm_kernel<kGmBf16, 128, 1, kGmRows, true, LGN_BF16>(), gm_kernel<kGmBf16, 128, 1, kGmRows, true, LGN_F32>(),
        gm_kernel<kGmBf16, 32, 1, kGmSwap, true, LGN_BF16>(), gm_kernel<kGmBf16, 32, 1, kGmSwap, true, LGN_F32>(),
        gm_kernel<kGmBf16, 64, 1, kGmSwap, true, LGN_BF16>(), gm_kernel<kGmBf16, 64, 1, kGmSwap, true, LGN_F32>()};
    return {table, (int)(sizeof table / sizeof table[0])};
}

}  // namespace lgn
