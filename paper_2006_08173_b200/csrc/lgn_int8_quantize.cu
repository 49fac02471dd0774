// Quantiser of matrices to 8-bit integers with one scale per row: the operands of lgn_int8_matmul.
//
// With a the largest magnitude of a row (2^-110 if that is larger) the scale is fl(a / 127), and the code of x is
// x fl(127 / a) rounded to nearest even.  One fused multiply-add onto 1.5 2^23 does that: its sum has a unit in the last
// place of 1, so the exact product is rounded to a whole number, once, and the number stands in the low bits.
// |x| <= a makes the product at most 127 (1 + 2^-24): no clamping.  2^-110 keeps 127 / a finite and a / 127 normal.
// A row with an entry that is not finite has a scale of NaN, which every product with it shows.
//
// The floor is memory: 2 or 4 bytes read and 1 written per value.  A row stays in registers between
// its maximum and its codes: 8 pieces of 16 bytes per thread, a warp or a CTA of 8 warps per row; longer rows are read again.
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_fp8.cuh"
#include "lgn_launch.h"
#include "lgn_log.h"
#include "lgn_values.cuh"

namespace lgn {

constexpr int kI8Pieces = 8;

// GROUP threads per row: 32, or the 256 of a CTA.
template <int DT, int GROUP, bool VEC>
__global__ void __launch_bounds__(256)
int8_rows_kernel(const char *x, uint64_t ld, uint32_t rows, uint32_t cols, int8_t *codes, uint32_t pitch, float *scales) {
    constexpr int ES = DT == LGN_F32 ? 4 : 2, N = 16 / ES;
    constexpr uint32_t kChunk = GROUP * N * kI8Pieces;
    __shared__ uint32_t wmax[8];
    dep_launch();
    dep_wait();
    const uint32_t lane = threadIdx.x % GROUP;
    const uint64_t row = (uint64_t)blockIdx.x * (256 / GROUP) + threadIdx.x / GROUP;
    if (row >= rows) return;                              // whole warps or the whole CTA
    const char *src = x + row * ld * ES;
    Values<DT, N> v[kI8Pieces];
    auto load = [&](uint32_t c0) {
        #pragma unroll
        for (int i = 0; i < kI8Pieces; ++i) {
            const uint64_t c = (uint64_t)c0 + (i * GROUP + lane) * N;
            v[i].template load<VEC>(src + c * ES, c < cols ? (int)min((uint64_t)N, cols - c) : 0);
        }
    };
    uint32_t a = 0;
    uint64_t c0 = 0;
    for (;;) {
        load((uint32_t)c0);
        #pragma unroll
        for (int i = 0; i < kI8Pieces; ++i) a = max(a, v[i].max_abs());
        c0 += kChunk;
        if (c0 >= pitch) break;
    }
    a = __reduce_max_sync(0xffffffffu, a);
    if constexpr (GROUP > 32) {
        if ((threadIdx.x & 31) == 0) wmax[threadIdx.x >> 5] = a;
        __syncthreads();
        #pragma unroll
        for (int w = 0; w < 8; ++w) a = max(a, wmax[w]);
    }
    const bool finite = a < 0x7f800000u;
    const float top = fmaxf(__uint_as_float(a), 7.7037197775489434e-34f);       // 2^-110
    const float per = finite ? __fdiv_rn(127.0f, top) : 0.0f;
    if (lane == 0) scales[row] = finite ? __fdiv_rn(top, 127.0f) : __int_as_float(0x7fffffff);
    int8_t *dst = codes + row * pitch;
    const bool held = pitch <= kChunk;                      // the one chunk is still in registers
    for (c0 = 0; c0 < pitch; c0 += kChunk) {
        if (!held) load((uint32_t)c0);
        #pragma unroll
        for (int i = 0; i < kI8Pieces; ++i) {
            const uint64_t c = c0 + (i * GROUP + lane) * N;
            if (c >= pitch) continue;
            uint32_t q[N / 4];
            #pragma unroll
            for (int k = 0; k < N / 4; ++k) {
                uint32_t w[4];
                #pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(fmaf(v[i].at(4 * k + j), per, 12582912.0f));
                q[k] = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
            }
            if constexpr (N == 8) *reinterpret_cast<uint2 *>(dst + c) = make_uint2(q[0], q[1]);
            else *reinterpret_cast<uint32_t *>(dst + c) = q[0];
        }
    }
}

#define LGN_I8(D, G, V) reinterpret_cast<const void *>(&int8_rows_kernel<D, G, V>)
static const void *const kInt8Table[2][2][2] = {{{LGN_I8(LGN_F32, 32, false), LGN_I8(LGN_F32, 32, true)}, {LGN_I8(LGN_F32, 256, false), LGN_I8(LGN_F32, 256, true)}},
                                                {{LGN_I8(LGN_BF16, 32, false), LGN_I8(LGN_BF16, 32, true)}, {LGN_I8(LGN_BF16, 256, false), LGN_I8(LGN_BF16, 256, true)}}};
#undef LGN_I8

}  // namespace lgn

using namespace lgn;

extern "C" size_t lgn_int8_codes_bytes(uint64_t rows, uint64_t cols) {
    if (rows > kFp8MaxDim || cols > kFp8MaxDim) return 0;
    return (size_t)(rows * fp8_pitch(cols));
}

extern "C" lgn_status lgn_int8_quantize(const void *x, uint64_t rows, uint64_t cols, uint64_t ld, lgn_dtype dt,
                                        void *codes, float *scales, void *stream) {
    if (dt != LGN_F32 && dt != LGN_BF16) return LGN_ERR_INVALID_ARG;
    if (rows > kFp8MaxDim || cols > kFp8MaxDim) return LGN_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return LGN_OK;
    if (ld < cols || ld > (1ull << 40)) return LGN_ERR_INVALID_ARG;
    const uint64_t es = dt == LGN_F32 ? 4 : 2, xb = matrix_bytes(rows, cols, ld, es), qb = lgn_int8_codes_bytes(rows, cols);
    if (xb == 0 || x == nullptr || codes == nullptr || scales == nullptr) return LGN_ERR_INVALID_ARG;
    if (!aligned_to(x, es) || !aligned_to(codes, 16) || !aligned_to(scales, 4)) return LGN_ERR_INVALID_ARG;
    if (ranges_overlap(x, xb, codes, qb) || ranges_overlap(x, xb, scales, 4 * rows) || ranges_overlap(codes, qb, scales, 4 * rows)) return LGN_ERR_INVALID_ARG;
    const bool vec = aligned_to(x, 16) && (ld * es) % 16 == 0;
    uint32_t r = (uint32_t)rows, c = (uint32_t)cols, pitch = (uint32_t)fp8_pitch(cols);
    // a CTA per row where a warp would not hold it, and where warps per row would leave SMs without one
    const uint64_t warp_cols = 32 * (16 / es) * kI8Pieces;
    const bool wide = cols > warp_cols || (rows < 148 * 4 && cols > 256);
    const uint64_t ctas = wide ? rows : (rows + 7) / 8;
    log_line("int8_quantize: rows %u cols %u, %s per row", r, c, wide ? "a CTA" : "a warp");
    void *args[] = {&x, &ld, &r, &c, &codes, &pitch, &scales};
    return launch_dependent(kInt8Table[dt][wide][vec], dim3((unsigned)ctas), dim3(256), args, 0, stream);
}
