// Instances of the grouped product: dY^T X over each group's rows in bf16 (weight gradients).
#include "lgn_grouped.cuh"

namespace lgn {

GmKernels gm_weight_kernels() {
    static const GmKernel table[] = {
        gm_kernel<kGmBf16, 256, 2, kGmGrad, false, LGN_BF16>(), gm_kernel<kGmBf16, 256, 2, kGmGrad, false, LGN_F32>(),
        gm_kernel<kGmBf16, 128, 1, kGmGrad, false, LGN_BF16>(), gm_kernel<kGmBf16, 128, 1, kGmGrad, false, LGN_F32>(),
        gm_kernel<kGmBf16, 128, 1, kGmShare, false, LGN_BF16>(), gm_kernel<kGmBf16, 128, 1, kGmShare, false, LGN_F32>()};
    return {table, (int)(sizeof table / sizeof table[0])};
}

}  // namespace lgn
