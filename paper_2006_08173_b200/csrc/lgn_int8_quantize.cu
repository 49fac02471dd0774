// Quantiser of matrices to 8-bit integers with one scale per row: the operands of lgn_int8_matmul.
//
// With a the largest magnitude of a row (2^-110 if that is larger) the scale is fl(a / 127), and the code of x is
// x fl(127 / a) rounded to nearest even.  One fused multiply-add onto 1.5 2^23 does that: its sum has a unit in the last
// place of 1, so the exact product is rounded to a whole number, once, and the number stands in the low bits.
// |x| <= a makes the product at most 127 (1 + 2^-24): no clamping.  2^-110 keeps 127 / a finite and a / 127 normal.
// A row with an entry that is not finite has a scale of NaN, which every product with it shows.
//
// The floor is memory: 2 or 4 bytes read and 1 written per value.  A row stays in registers between
// its maximum and its codes: 8 pieces of 16 bytes per thread, 1, 2, 4 or 8 warps per row; longer rows are read again.  The fewest warps that hold a row
// are taken (8192 x 4096 bf16: 2 warps 16.6 us, 8 warps 40 us: most of their registers are empty), more where there are few rows.
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_fp8.cuh"
#include "lgn_launch.h"
#include "lgn_log.h"
#include "lgn_values.cuh"

namespace lgn {

constexpr int kI8Pieces = 8;

// GROUP threads per row; 256 / GROUP rows per CTA.
template <int DT, int GROUP, bool VEC>
__global__ void __launch_bounds__(256)
int8_rows_kernel(const char *x, uint64_t ld, uint32_t rows, uint32_t cols, int8_t *codes, uint32_t pitch, float *scales) {
    constexpr int ES = DT == LGN_F32 ? 4 : 2, N = 16 / ES;
    constexpr uint32_t kPiece = GROUP * N, kChunk = kPiece * kI8Pieces;
    __shared__ uint32_t wmax[8];
    dep_launch();
    dep_wait();
    const uint32_t lane = threadIdx.x % GROUP;
    const uint64_t row = (uint64_t)blockIdx.x * (256 / GROUP) + threadIdx.x / GROUP;
    const bool live = row < rows;                         // the same for a row's warps
    const char *src = x + row * ld * ES;
    Values<DT, N> v[kI8Pieces];
    auto load = [&](uint64_t c0) {
        #pragma unroll
        for (int i = 0; i < kI8Pieces; ++i) {
            if (c0 + i * kPiece >= pitch) break;          // pieces that no thread of the row has
            const uint64_t c = c0 + i * kPiece + lane * N;
            v[i].template load<VEC>(src + c * ES, c < cols ? (int)min((uint64_t)N, cols - c) : 0);
        }
    };
    uint32_t a = 0;
    if (live) {
        for (uint64_t c0 = 0; c0 < pitch; c0 += kChunk) {
            load(c0);
            #pragma unroll
            for (int i = 0; i < kI8Pieces; ++i) {
                if (c0 + i * kPiece >= pitch) break;
                a = max(a, v[i].max_abs());
            }
        }
    }
    a = __reduce_max_sync(0xffffffffu, a);
    if constexpr (GROUP > 32) {
        if ((threadIdx.x & 31) == 0) wmax[threadIdx.x >> 5] = a;
        __syncthreads();
        const uint32_t first = threadIdx.x / GROUP * (GROUP / 32);
        #pragma unroll
        for (int w = 0; w < GROUP / 32; ++w) a = max(a, wmax[first + w]);
    }
    if (!live) return;
    const bool finite = a < 0x7f800000u;
    const float top = fmaxf(__uint_as_float(a), 7.7037197775489434e-34f);       // 2^-110
    const float per = finite ? __fdiv_rn(127.0f, top) : 0.0f;
    if (lane == 0) scales[row] = finite ? __fdiv_rn(top, 127.0f) : __int_as_float(0x7fffffff);
    int8_t *dst = codes + row * pitch;
    const bool held = pitch <= kChunk;                      // the one chunk is still in registers
    for (uint64_t c0 = 0; c0 < pitch; c0 += kChunk) {
        if (!held) load(c0);
        #pragma unroll
        for (int i = 0; i < kI8Pieces; ++i) {
            const uint64_t c = c0 + i * kPiece + lane * N;
            if (c >= pitch) break;
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
#define LGN_I8G(D, G) {LGN_I8(D, G, false), LGN_I8(D, G, true)}
static const void *const kInt8Table[2][4][2] = {{LGN_I8G(LGN_F32, 32), LGN_I8G(LGN_F32, 64), LGN_I8G(LGN_F32, 128), LGN_I8G(LGN_F32, 256)},
                                                {LGN_I8G(LGN_BF16, 32), LGN_I8G(LGN_BF16, 64), LGN_I8G(LGN_BF16, 128), LGN_I8G(LGN_BF16, 256)}};
#undef LGN_I8G
#undef LGN_I8

// ------------------------------------------------------------------ rows of whole 16-byte pieces
// One thread per piece: 8 values at any 2-byte boundary, read one by one (the lanes of a warp read the same lines), zeros behind the last column.
__global__ void __launch_bounds__(256)
align_rows_kernel(const char *x, uint64_t ld, uint64_t group, uint64_t rows, uint32_t cols, uint32_t pieces, uint64_t total, uint4 *out) {
    dep_launch();
    dep_wait();
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / pieces;
        const uint32_t c = (uint32_t)(i - row * pieces) * 8;
        const uint64_t g = row / rows;
        const char *src = x + (g * group + (row - g * rows) * ld + c) * 2;
        uint32_t w[4];
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = c + 2 * k < cols ? ldro_u16(src + 4 * k) : 0u;
            if (c + 2 * k + 1 < cols) w[k] |= ldro_u16(src + 4 * k + 2) << 16;
        }
        out[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

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
    if (rows == 0 || (cols == 0 && scales == nullptr)) return LGN_OK;
    const uint64_t es = dt == LGN_F32 ? 4 : 2;
    if (!aligned_to(scales, 4)) return LGN_ERR_INVALID_ARG;
    if (cols > 0) {                                         // rows without a column have scales, and nothing to read
        if (ld < cols || ld > (1ull << 40)) return LGN_ERR_INVALID_ARG;
        const uint64_t xb = matrix_bytes(rows, cols, ld, es), qb = lgn_int8_codes_bytes(rows, cols);
        if (xb == 0 || x == nullptr || codes == nullptr || scales == nullptr) return LGN_ERR_INVALID_ARG;
        if (!aligned_to(x, es) || !aligned_to(codes, 16)) return LGN_ERR_INVALID_ARG;
        if (ranges_overlap(x, xb, codes, qb) || ranges_overlap(x, xb, scales, 4 * rows) || ranges_overlap(codes, qb, scales, 4 * rows)) return LGN_ERR_INVALID_ARG;
    }
    const bool vec = aligned_to(x, 16) && (ld * es) % 16 == 0;
    uint32_t r = (uint32_t)rows, c = (uint32_t)cols, pitch = (uint32_t)fp8_pitch(cols);
    // the fewest warps that hold a row; twice as many for as long as the SMs have fewer than four each and every thread has a piece
    const uint64_t piece = 16 / es;
    int group = 0;
    while (group < 3 && (cols > (32ull << group) * piece * kI8Pieces || ((rows << group) < 148 * 4 && cols >= (64ull << group) * piece))) ++group;
    const uint64_t per_cta = 8u >> group, ctas = (rows + per_cta - 1) / per_cta;
    log_line("int8_quantize: rows %u cols %u, %d warps per row", r, c, 1 << group);
    void *args[] = {&x, &ld, &r, &c, &codes, &pitch, &scales};
    return launch_dependent(kInt8Table[dt][group][vec], dim3((unsigned)ctas), dim3(256), args, 0, stream);
}

extern "C" lgn_status lgn_align_rows(const void *x, uint64_t ld, uint64_t x_group, uint64_t groups, uint64_t rows, uint64_t cols, void *out, void *stream) {
    if (rows > kFp8MaxDim || cols > kFp8MaxDim || groups > (1ull << 20)) return LGN_ERR_UNSUPPORTED;
    if (groups == 0 || rows == 0 || cols == 0) return LGN_OK;
    if (ld < cols || ld > (1ull << 40) || (groups > 1 && x_group > (1ull << 40))) return LGN_ERR_INVALID_ARG;
    const uint64_t one = matrix_bytes(rows, cols, ld, 2), pieces = (cols + 7) / 8;
    if (one == 0 || x == nullptr || out == nullptr || !aligned_to(x, 2) || !aligned_to(out, 16)) return LGN_ERR_INVALID_ARG;
    if (groups > 1 && groups - 1 > ((1ull << 60) - one) / (2 * (x_group > 0 ? x_group : 1))) return LGN_ERR_INVALID_ARG;
    if (rows * pieces > (1ull << 58) / groups) return LGN_ERR_INVALID_ARG;
    const uint64_t total = groups * rows * pieces;
    if (ranges_overlap(x, (groups - 1) * x_group * 2 + one, out, total * 16)) return LGN_ERR_INVALID_ARG;
    uint32_t c = (uint32_t)cols, p = (uint32_t)pieces;
    uint64_t t = total;
    const uint64_t want = (total + 255) / 256;
    void *args[] = {&x, &ld, &x_group, &rows, &c, &p, &t, &out};
    return launch_dependent(reinterpret_cast<const void *>(&align_rows_kernel), dim3((unsigned)(want < (1u << 20) ? want : 1u << 20)), dim3(256), args, 0, stream);
}
