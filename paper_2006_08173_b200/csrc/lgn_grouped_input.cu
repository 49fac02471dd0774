// Instances of the grouped product: X W_e in bf16 (input gradients).
#include "lgn_grouped.cuh"

namespace lgn {

GmKernels gm_input_kernels() {
    static const GmKernel table[] = {
        gm_kernel<kGmBf16, 256, 2, kGmTurn, false, LGN_BF16>(), gm_kernel<kGmBf16, 256, 2, kGmTurn, false, LGN_F32>(),
        gm_kernel<kGmBf16, 256, 2, kGmRows, false, LGN_BF16>(), gm_kernel<kGmBf16, 256, 2, kGmRows, false, LGN_F32>(),
        gm_kernel<kGmBf16, 128, 1, kGmRows, false, LGN_BF16>(), gm_kernel<kGmBf16, 128, 1, kGmRows, false, LGN_F32>(),
        gm_kernel<kGmBf16, 32, 1, kGmSwap, false, LGN_BF16>(), gm_kernel<kGmBf16, 32, 1, kGmSwap, false, LGN_F32>(),
        gm_kernel<kGmBf16, 64, 1, kGmSwap, false, LGN_BF16>(), gm_kernel<kGmBf16, 64, 1, kGmSwap, false, LGN_F32>()};
    return {table, (int)(sizeof table / sizeof table[0])};
}

}  // namespace lgn
