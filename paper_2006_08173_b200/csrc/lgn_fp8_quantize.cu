// Quantiser of matrices to 8-bit floating point (E4M3, E5M2) with one power-of-two scale per
// block of 128 values: the operands of lgn_fp8_matmul.
//
// A block's exponent e is the smallest integer >= -127 with max|x| 2^-e <= f_max (f_max = 448 or
// 57344, both 1.75 2^k), taken over the block's finite entries; the codes are x 2^-e rounded to
// nearest even.  With max|x| = m 2^E, 1 <= m < 2, that is e = E - k + (m > 1.75): two integer
// operations on the fp32 pattern.  x 2^-e is exact unless it falls below the smallest normal fp32
// number, far below half of the smallest code, so each code is rounded once.
//
// The floor is memory: 2 or 4 bytes read and 1 (or, with the transposed copy, 2) written per value.  What comes nearer to its limit is the
// integer pipe, 62 % busy for rows, 77 % for both copies (8192 x 4096 bf16, DRAM at 41 and 29 %).
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_fp8.cuh"
#include "lgn_launch.h"
#include "lgn_log.h"

namespace lgn {

// Pattern of |x| if x is finite, else 0.
__device__ __forceinline__ uint32_t finite_abs(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// Biased exponent e + 127 (the E8M0 byte) of a block whose largest finite magnitude has pattern a.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
    const int e = (int)(a >> 23) - (FMT == LGN_E4M3 ? 8 : 15) + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);      // + 127 - 127
    return (uint32_t)max(e, 0);
}

// Pattern of 2^-e for a biased exponent 0..247.
__device__ __forceinline__ uint32_t inverse_scale(uint32_t byte) { return (254u - byte) << 23; }

template <int FMT>
__device__ __forceinline__ uint32_t code_pair(float lo, float hi) {                   // two codes, lo in bits 0..7
    uint16_t r;
    if constexpr (FMT == LGN_E4M3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else                           asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int FMT>
__device__ __forceinline__ uint32_t code_quad(float a, float b, float c, float d) {
    return __byte_perm(code_pair<FMT>(a, b), code_pair<FMT>(c, d), 0x5410);
}

// Every non-finite x becomes NaN (the saturating conversion would store an infinity as the largest
// code; the NaN code keeps it visible in every sum it takes part in).
__device__ __forceinline__ float nan_if_not_finite(float x) {
    return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? __int_as_float(0x7fffffff) : x;
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Two bf16 values times two powers of two: exact above the subnormals.
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {                          // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// N consecutive values of a row as they lie in memory: N words of fp32, N/2 of two bf16 each.  A value costs
// about six instructions per copy written, so bf16 stays packed for maxima and scaling.
template <int DT, int N> struct Values {
    static constexpr int kWords = DT == LGN_F32 ? N : N / 2;
    uint32_t w[kWords];

    // of which the first `valid` exist (others read as 0)
    template <bool VEC>
    __device__ __forceinline__ void load(const char *p, int valid) {
        if (VEC && valid >= N) {
            #pragma unroll
            for (int k = 0; k < kWords; k += 4)
                asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3]) : "l"(p + 4 * k) : "memory");
            return;
        }
        #pragma unroll
        for (int k = 0; k < kWords; ++k) {
            w[k] = 0u;
            if constexpr (DT == LGN_F32) {
                if (k < valid) w[k] = ldro_u32(p + 4 * k);
            } else {
                if (2 * k < valid) w[k] = ldro_u16(p + 4 * k);
                if (2 * k + 1 < valid) w[k] |= ldro_u16(p + 4 * k + 2) << 16;
            }
        }
    }
    __device__ __forceinline__ float at(int k) const {
        if constexpr (DT == LGN_F32) return __uint_as_float(w[k]);
        else return k & 1 ? bf_hi(w[k >> 1]) : bf_lo(w[k >> 1]);
    }
    // fp32 pattern of the largest magnitude: at least 0x7f800000 if any value is not finite
    __device__ __forceinline__ uint32_t max_abs() const {
        if constexpr (DT == LGN_F32) {
            float m = fabsf(__uint_as_float(w[0]));
            #pragma unroll
            for (int k = 1; k < kWords; ++k) m = max_nan(m, fabsf(__uint_as_float(w[k])));
            return __float_as_uint(m) & 0x7fffffffu;
        } else {
            uint32_t m = w[0] & 0x7fff7fffu;
            #pragma unroll
            for (int k = 1; k < kWords; ++k) m = __vmaxu2(m, w[k] & 0x7fff7fffu);
            return max(m << 16, m & 0xffff0000u);
        }
    }
    __device__ __forceinline__ uint32_t max_abs_finite() const {
        uint32_t a = 0;
        #pragma unroll
        for (int k = 0; k < N; ++k) a = max(a, finite_abs(at(k)));
        return a;
    }
    // codes of values 4q .. 4q + 3, all with the scale whose inverse has pattern inv
    template <int FMT>
    __device__ __forceinline__ uint32_t quad(int q, uint32_t inv, bool special) const {
        if (special) {
            const float f = __uint_as_float(inv);
            return code_quad<FMT>(nan_if_not_finite(at(4 * q)) * f, nan_if_not_finite(at(4 * q + 1)) * f,
                                  nan_if_not_finite(at(4 * q + 2)) * f, nan_if_not_finite(at(4 * q + 3)) * f);
        }
        if constexpr (DT == LGN_F32) {
            const float f = __uint_as_float(inv);
            return code_quad<FMT>(at(4 * q) * f, at(4 * q + 1) * f, at(4 * q + 2) * f, at(4 * q + 3) * f);
        } else {
            const uint32_t f = __byte_perm(inv, inv, 0x3232), a = mul_bf16x2(w[2 * q], f), b = mul_bf16x2(w[2 * q + 1], f);
            return code_quad<FMT>(bf_lo(a), bf_hi(a), bf_lo(b), bf_hi(b));
        }
    }
};

// ------------------------------------------------------------------ row blocks only
// One warp takes 512 consecutive columns of one row, 16 per lane: a block of 128 lies in 8 lanes
// (three shuffles for its maximum), a lane writes its 16 codes at once and the warp's four scales
// are one word of the scale tile.
template <int DT, int FMT, bool VEC>
__global__ void __launch_bounds__(256)
fp8_rows_kernel(const char *x, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t groups,
                uint8_t *codes, uint32_t ldq, uint32_t *scales) {
    dep_launch();
    dep_wait();
    constexpr int ES = DT == LGN_F32 ? 4 : 2;
    const uint64_t unit = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t row = (uint32_t)(unit / groups), grp = (uint32_t)(unit % groups);
    if (row >= rows) return;
    const uint32_t c0 = grp * 512 + lane * 16;
    Values<DT, 16> v;
    v.template load<VEC>(x + ((uint64_t)row * ld + c0) * ES, (int)min((int64_t)16, (int64_t)cols - (int64_t)c0));
    uint32_t a = v.max_abs();
    const bool special = __any_sync(0xffffffffu, a >= 0x7f800000u);
    if (special) a = v.max_abs_finite();
    #pragma unroll
    for (int d = 1; d < 8; d <<= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, d));
    const uint32_t byte = scale_byte<FMT>(a), inv = inverse_scale(byte);
    if (c0 < ldq) {
        uint4 q;
        q.x = v.template quad<FMT>(0, inv, special); q.y = v.template quad<FMT>(1, inv, special);
        q.z = v.template quad<FMT>(2, inv, special); q.w = v.template quad<FMT>(3, inv, special);
        *reinterpret_cast<uint4 *>(codes + (uint64_t)row * ldq + c0) = q;
    }
    uint32_t word = byte << (8 * (lane >> 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    word |= __shfl_xor_sync(0xffffffffu, word, 16);
    if (lane == 0) scales[fp8_scale_word(row, grp, groups)] = word;
}

// ------------------------------------------------------------------ 128 x 128 tiles
// Transposed copies and square blocks.  A CTA keeps its tile in registers (thread: 8 consecutive
// rows x 8 consecutive columns), so the tile is read once for both copies.  Maxima go through shared memory:
// every thread leaves its 8 row and 8 column maxima, then one thread per row and one per column adds up 16 of
// them and forms the scale.  Transposed codes leave through shared memory as units of 8 bytes (8 rows of one column);
// unit u of column c sits at place u ^ (c / 8), which spreads the 16 lanes that write units of columns 8
// apart over all banks.
// BLOCKS: blocks of 128 along the rows of both copies, of the transpose alone, or squares.
enum TileBlocks { kTileBoth = 0, kTileTransposed = 1, kTileSquare = 2 };
// Four CTAs per SM (64 registers, 12 bytes of them spilled with both copies) hide the latency of the loads and of the shared
// tile: both bf16 copies of 16384 x 8192 take 139, 126 and 115 us with two, three and four.  fp32 holds twice the values
// per thread, so two fit without spills.
template <int DT, int FMT, int BLOCKS, bool VEC>
__global__ void __launch_bounds__(256, DT == LGN_F32 ? 2 : 4)
fp8_tile_kernel(const char *x, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t col_tiles,
                uint8_t *codes, uint32_t ldq, uint8_t *scales, uint32_t groups,
                uint8_t *codes_t, uint32_t ldq_t, uint8_t *scales_t, uint32_t groups_t) {
    __shared__ __align__(16) uint2 tr[128 * 16];
    __shared__ uint32_t rmax[128 * 17];
    __shared__ __align__(16) uint32_t cmax[16 * 128];
    __shared__ uint32_t rinv[128];
    __shared__ __align__(16) uint32_t cinv[128];
    __shared__ uint32_t wmax[8];
    constexpr bool SQUARE = BLOCKS == kTileSquare, ROWS = BLOCKS == kTileBoth, COLS = BLOCKS != kTileSquare;
    dep_launch();
    dep_wait();
    constexpr int ES = DT == LGN_F32 ? 4 : 2;
    const uint32_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
    const uint32_t cg = threadIdx.x & 15, rg = threadIdx.x >> 4, cl = cg * 8, rl = rg * 8;          // within the tile
    const uint32_t c0 = ct * 128 + cl, r0 = rt * 128 + rl;
    Values<DT, 8> v[8];
    const int valid = (int)min((int64_t)8, (int64_t)cols - (int64_t)c0);
    #pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i].template load<VEC>(x + ((uint64_t)(r0 + i) * ld + c0) * ES, r0 + i < rows ? valid : 0);

    bool special = false;
    for (int round = 0; round < 2; ++round) {             // a second round, over finite values, only where some are not
        uint32_t mine = 0;
        if constexpr (SQUARE || ROWS) {
            #pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t a = special ? v[i].max_abs_finite() : v[i].max_abs();
                if constexpr (SQUARE) mine = max(mine, a);
                else rmax[(rl + i) * 17 + cg] = a;
            }
        }
        if constexpr (SQUARE) {
            mine = __reduce_max_sync(0xffffffffu, mine);
            if ((threadIdx.x & 31) == 0) wmax[threadIdx.x >> 5] = mine;
        }
        if constexpr (COLS) {
            uint32_t m[8];
            if (special) {
                #pragma unroll
                for (int j = 0; j < 8; ++j) {
                    m[j] = 0u;
                    #pragma unroll
                    for (int i = 0; i < 8; ++i) m[j] = max(m[j], finite_abs(v[i].at(j)));
                }
            } else if constexpr (DT == LGN_F32) {
                #pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float f = fabsf(v[0].at(j));
                    #pragma unroll
                    for (int i = 1; i < 8; ++i) f = max_nan(f, fabsf(v[i].at(j)));
                    m[j] = __float_as_uint(f) & 0x7fffffffu;
                }
            } else {
                #pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t t = v[0].w[q] & 0x7fff7fffu;
                    #pragma unroll
                    for (int i = 1; i < 8; ++i) t = __vmaxu2(t, v[i].w[q] & 0x7fff7fffu);
                    m[2 * q] = t << 16;
                    m[2 * q + 1] = t & 0xffff0000u;
                }
            }
            *reinterpret_cast<uint4 *>(&cmax[rg * 128 + cl]) = make_uint4(m[0], m[1], m[2], m[3]);
            *reinterpret_cast<uint4 *>(&cmax[rg * 128 + cl + 4]) = make_uint4(m[4], m[5], m[6], m[7]);
        }
        __syncthreads();
        const uint32_t t = threadIdx.x & 127;
        const bool is_col = threadIdx.x >= 128;
        uint32_t a = 0;
        if constexpr (SQUARE) {
            #pragma unroll
            for (int k = 0; k < 8; ++k) a = max(a, wmax[k]);
        } else if (is_col) {
            #pragma unroll
            for (int k = 0; k < 16; ++k) a = max(a, cmax[k * 128 + t]);
        } else if constexpr (ROWS) {
            #pragma unroll
            for (int k = 0; k < 16; ++k) a = max(a, rmax[t * 17 + k]);
        }
        if (round == 0) {
            special = __syncthreads_or(a >= 0x7f800000u);
            if (special) continue;
        }
        const uint32_t byte = scale_byte<FMT>(a);
        if (is_col) {
            cinv[t] = inverse_scale(byte);
            if (codes_t != nullptr) scales_t[4 * fp8_scale_word(ct * 128 + t, rt >> 2, groups_t) + (rt & 3)] = (uint8_t)byte;
        } else {
            rinv[t] = inverse_scale(byte);
            if (BLOCKS != kTileTransposed && codes != nullptr) scales[4 * fp8_scale_word(rt * 128 + t, ct >> 2, groups) + (ct & 3)] = (uint8_t)byte;
        }
        break;
    }
    __syncthreads();
    if (!(BLOCKS == kTileTransposed) && codes != nullptr && c0 < ldq) {                                               // ldq is a multiple of 16
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t inv = rinv[rl + i];
            if (r0 + i < rows)
                *reinterpret_cast<uint2 *>(codes + (uint64_t)(r0 + i) * ldq + c0) =
                    make_uint2(v[i].template quad<FMT>(0, inv, special), v[i].template quad<FMT>(1, inv, special));
        }
    }
    if (codes_t != nullptr) {
        #pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const uint2 inv = *reinterpret_cast<const uint2 *>(&cinv[cl + j]);
            float lo[8], hi[8];
            if (DT == LGN_F32 || special) {
                #pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float a = v[i].at(j), b = v[i].at(j + 1);
                    lo[i] = (special ? nan_if_not_finite(a) : a) * __uint_as_float(inv.x);
                    hi[i] = (special ? nan_if_not_finite(b) : b) * __uint_as_float(inv.y);
                }
            } else {
                const uint32_t f = __byte_perm(inv.x, inv.y, 0x7632);
                #pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t y = mul_bf16x2(v[i].w[j / 2], f);
                    lo[i] = bf_lo(y);
                    hi[i] = bf_hi(y);
                }
            }
            tr[(cl + j) * 16 + (rg ^ cg)] = make_uint2(code_quad<FMT>(lo[0], lo[1], lo[2], lo[3]), code_quad<FMT>(lo[4], lo[5], lo[6], lo[7]));
            tr[(cl + j + 1) * 16 + (rg ^ cg)] = make_uint2(code_quad<FMT>(hi[0], hi[1], hi[2], hi[3]), code_quad<FMT>(hi[4], hi[5], hi[6], hi[7]));
        }
        __syncthreads();
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t id = k * 256 + threadIdx.x, c = id >> 3, u = (id & 7) * 2, sw = (c >> 3) & 15;
            const uint2 a = tr[c * 16 + (u ^ sw)], b = tr[c * 16 + ((u + 1) ^ sw)];
            const uint32_t gc = ct * 128 + c, gr = rt * 128 + u * 8;
            if (gc < cols && gr < ldq_t)
                *reinterpret_cast<uint4 *>(codes_t + (uint64_t)gc * ldq_t + gr) = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
}

#define LGN_ROWS(D, F, V) reinterpret_cast<const void *>(&fp8_rows_kernel<D, F, V>)
static const void *const kRowsTable[2][2][2] = {
    {{LGN_ROWS(LGN_F32, LGN_E4M3, false), LGN_ROWS(LGN_F32, LGN_E4M3, true)}, {LGN_ROWS(LGN_F32, LGN_E5M2, false), LGN_ROWS(LGN_F32, LGN_E5M2, true)}},
    {{LGN_ROWS(LGN_BF16, LGN_E4M3, false), LGN_ROWS(LGN_BF16, LGN_E4M3, true)}, {LGN_ROWS(LGN_BF16, LGN_E5M2, false), LGN_ROWS(LGN_BF16, LGN_E5M2, true)}}};
#undef LGN_ROWS
#define LGN_TILE(D, F, S, V) reinterpret_cast<const void *>(&fp8_tile_kernel<D, F, S, V>)
#define LGN_TILE4(D, F) {{LGN_TILE(D, F, kTileBoth, false), LGN_TILE(D, F, kTileBoth, true)}, {LGN_TILE(D, F, kTileTransposed, false), LGN_TILE(D, F, kTileTransposed, true)}, \
                         {LGN_TILE(D, F, kTileSquare, false), LGN_TILE(D, F, kTileSquare, true)}}
static const void *const kTileTable[2][2][3][2] = {{LGN_TILE4(LGN_F32, LGN_E4M3), LGN_TILE4(LGN_F32, LGN_E5M2)},
                                                   {LGN_TILE4(LGN_BF16, LGN_E4M3), LGN_TILE4(LGN_BF16, LGN_E5M2)}};
#undef LGN_TILE4
#undef LGN_TILE

}  // namespace lgn

using namespace lgn;

extern "C" size_t lgn_fp8_codes_bytes(uint64_t rows, uint64_t cols) {
    if (rows > kFp8MaxDim || cols > kFp8MaxDim) return 0;
    return (size_t)(rows * fp8_pitch(cols));
}

extern "C" size_t lgn_fp8_scales_bytes(uint64_t rows, uint64_t cols) {
    if (rows > kFp8MaxDim || cols > kFp8MaxDim) return 0;
    return (size_t)(((rows + 127) / 128) * ((cols + 511) / 512) * 512);
}

extern "C" lgn_status lgn_fp8_quantize(const void *x, uint64_t rows, uint64_t cols, uint64_t ld, lgn_dtype dt,
                                       lgn_fp8 fmt, lgn_fp8_block block, void *codes, void *scales,
                                       void *codes_t, void *scales_t, void *stream) {
    if (dt != LGN_F32 && dt != LGN_BF16) return LGN_ERR_INVALID_ARG;
    if ((fmt != LGN_E4M3 && fmt != LGN_E5M2) || (block != LGN_BLOCK_ROW && block != LGN_BLOCK_SQUARE)) return LGN_ERR_INVALID_ARG;
    if (rows > kFp8MaxDim || cols > kFp8MaxDim) return LGN_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return LGN_OK;
    if (ld < cols || ld > (1ull << 40)) return LGN_ERR_INVALID_ARG;
    if (x == nullptr || !aligned_to(x, dt == LGN_F32 ? 4 : 2)) return LGN_ERR_INVALID_ARG;
    if ((codes == nullptr) != (scales == nullptr) || (codes_t == nullptr) != (scales_t == nullptr)) return LGN_ERR_INVALID_ARG;
    if (codes == nullptr && codes_t == nullptr) return LGN_ERR_INVALID_ARG;
    if (!aligned_to(codes, 16) || !aligned_to(scales, 16) || !aligned_to(codes_t, 16) || !aligned_to(scales_t, 16)) return LGN_ERR_INVALID_ARG;
    const uint64_t es = dt == LGN_F32 ? 4 : 2, xb = matrix_bytes(rows, cols, ld, es);
    if (xb == 0) return LGN_ERR_INVALID_ARG;
    struct { const void *p; uint64_t n; } b[5] = {
        {x, xb}, {codes, codes ? lgn_fp8_codes_bytes(rows, cols) : 0}, {scales, scales ? lgn_fp8_scales_bytes(rows, cols) : 0},
        {codes_t, codes_t ? lgn_fp8_codes_bytes(cols, rows) : 0}, {scales_t, scales_t ? lgn_fp8_scales_bytes(cols, rows) : 0}};
    for (int i = 0; i < 5; ++i)
        for (int j = i + 1; j < 5; ++j)
            if (ranges_overlap(b[i].p, b[i].n, b[j].p, b[j].n)) return LGN_ERR_INVALID_ARG;
    const bool vec = aligned_to(x, 16) && (ld * es) % 16 == 0;
    uint32_t r = (uint32_t)rows, c = (uint32_t)cols, ldq = (uint32_t)fp8_pitch(cols), ldq_t = (uint32_t)fp8_pitch(rows);
    uint32_t groups = (c + 511) / 512, groups_t = (r + 511) / 512;
    if (block == LGN_BLOCK_ROW && codes_t == nullptr) {
        const uint64_t blocks = ((uint64_t)r * groups + 7) / 8;
        if (blocks > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
        log_line("fp8_quantize: rows %u cols %u, row blocks, %llu CTAs", r, c, (unsigned long long)blocks);
        void *args[] = {&x, &ld, &r, &c, &groups, &codes, &ldq, &scales};
        return launch_dependent(kRowsTable[dt][fmt][vec], dim3((unsigned)blocks), dim3(256), args, 0, stream);
    }
    uint32_t col_tiles = (c + 127) / 128;
    const uint64_t tiles = (uint64_t)((r + 127) / 128) * col_tiles;
    if (tiles > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    log_line("fp8_quantize: rows %u cols %u, %s blocks, %llu tiles", r, c, block == LGN_BLOCK_SQUARE ? "square" : "row", (unsigned long long)tiles);
    void *args[] = {&x, &ld, &r, &c, &col_tiles, &codes, &ldq, &scales, &groups, &codes_t, &ldq_t, &scales_t, &groups_t};
    const int blocks = block == LGN_BLOCK_SQUARE ? kTileSquare : codes == nullptr ? kTileTransposed : kTileBoth;
    return launch_dependent(kTileTable[dt][fmt][blocks][vec], dim3((unsigned)tiles), dim3(256), args, 0, stream);
}
