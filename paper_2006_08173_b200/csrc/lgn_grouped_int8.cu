// Instances of the grouped product: X W_e^T in 8-bit integers.
#include "lgn_grouped.cuh"

namespace lgn {

GmKernels gm_int8_kernels() {
    static const GmKernel table[] = {
        gm_kernel<kGmInt8, 256, 2, kGmTurn, true, LGN_BF16>(), gm_kernel<kGmInt8, 256, 2, kGmTurn, true, LGN_F32>(),
        gm_kernel<kGmInt8, 256, 2, kGmRows, true, LGN_BF16>(), gm_kernel<kGmInt8, 256, 2, kGmRows, true, LGN_F32>(),
        gm_kernel<kGmInt8, 128, 2, kGmRows, true, LGN_BF16>(), gm_kernel<kGmInt8, 128, 2, kGmRows, true, LGN_F32>(),
        gm_kernel<kGmInt8, 128, 1, kGmRows, true, LGN_BF16>(), gm_kernel<kGmInt8, 128, 1, kGmRows, true, LGN_F32>(),
        gm_kernel<kGmInt8, 32, 1, kGmSwap, true, LGN_BF16>(), gm_kernel<kGmInt8, 32, 1, kGmSwap, true, LGN_F32>()};
    return {table, (int)(sizeof table / sizeof table[0])};
}

}  // namespace lgn
