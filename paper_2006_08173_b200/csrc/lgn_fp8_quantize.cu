// Quantiser of matrices to 8-bit floating point (E4M3, E5M2) with one power-of-two scale per
// block of 128 values: the operands of lgn_fp8_matmul.
//
// A block's exponent e is the smallest integer >= -127 with max|x| 2^-e <= f_max (f_max = 448 or
// 57344, both 1.75 2^k), taken over the block's finite entries; the codes are x 2^-e rounded to
// nearest even.  With max|x| = m 2^E, 1 <= m < 2, that is e = E - k + (m > 1.75): two integer
// operations on the fp32 pattern.  x 2^-e is exact unless it falls below the smallest normal fp32
// number, far below half of the smallest code, so each code is rounded once.
//
// Bound by memory: 2 or 4 bytes read and 1 (or, with the transposed copy, 2) written per value.
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
// `top` is 8 (E4M3) or 15 (E5M2).
__device__ __forceinline__ uint32_t scale_byte(uint32_t a, int top) {
    const int e = (int)(a >> 23) - top + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);      // + 127 - 127
    return (uint32_t)max(e, 0);
}

// 2^-e for a biased exponent 0..247.
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

template <int FMT>
__device__ __forceinline__ uint32_t code_pair(float lo, float hi) {                   // two codes, lo in bits 0..7
    uint16_t r;
    if constexpr (FMT == LGN_E4M3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else                           asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// x 2^-e with every non-finite x turned into NaN (the saturating conversion would store an infinity
// as the largest code; the NaN code keeps it visible in every sum it takes part in).
__device__ __forceinline__ float scaled(float x, float inv) {
    const float y = x * inv;
    return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? __int_as_float(0x7fffffff) : y;
}

template <int FMT>
__device__ __forceinline__ uint32_t code_quad(const float *x, float inv) {
    return code_pair<FMT>(scaled(x[0], inv), scaled(x[1], inv)) | code_pair<FMT>(scaled(x[2], inv), scaled(x[3], inv)) << 16;
}

// N consecutive values starting at p, of which the first `valid` exist (others read as 0).
template <int DT, int N, bool VEC>
__device__ __forceinline__ void load_values(const char *p, int valid, float *x) {
    if constexpr (VEC) {
        if (valid >= N) {
            if constexpr (DT == LGN_F32) {
                #pragma unroll
                for (int k = 0; k < N; k += 4) {
                    float4 v;
                    asm volatile("ld.global.nc.L1::no_allocate.v4.f32 {%0,%1,%2,%3}, [%4];"
                                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p + 4 * k));
                    x[k] = v.x; x[k + 1] = v.y; x[k + 2] = v.z; x[k + 3] = v.w;
                }
            } else {
                #pragma unroll
                for (int k = 0; k < N; k += 8) {
                    uint32_t w[4];
                    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p + 2 * k));
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[k + 2 * j] = __uint_as_float(w[j] << 16);
                        x[k + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                    }
                }
            }
            return;
        }
    }
    #pragma unroll
    for (int k = 0; k < N; ++k) {
        x[k] = 0.0f;
        if (k < valid) {
            if constexpr (DT == LGN_F32) x[k] = __uint_as_float(ldro_u32(p + 4 * k));
            else x[k] = __uint_as_float(ldro_u16(p + 2 * k) << 16);
        }
    }
}

// ------------------------------------------------------------------ row blocks only
// One warp takes 512 consecutive columns of one row, 16 per lane: a block of 128 lies in 8 lanes
// (three shuffles for its maximum), a lane writes its 16 codes at once and the warp's four scales
// are one word of the scale tile.
template <int DT, int FMT, bool VEC>
__global__ void __launch_bounds__(256)
fp8_rows_kernel(const char *__restrict__ x, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t groups,
                uint8_t *__restrict__ codes, uint32_t ldq, uint32_t *__restrict__ scales) {
    dep_launch();
    dep_wait();
    constexpr int ES = DT == LGN_F32 ? 4 : 2;
    const uint64_t unit = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t row = (uint32_t)(unit / groups), grp = (uint32_t)(unit % groups);
    if (row >= rows) return;
    const uint32_t c0 = grp * 512 + lane * 16;
    float v[16];
    load_values<DT, 16, VEC>(x + ((uint64_t)row * ld + c0) * ES, (int)min((int64_t)16, (int64_t)cols - (int64_t)c0), v);
    uint32_t a = 0;
    #pragma unroll
    for (int k = 0; k < 16; ++k) a = max(a, finite_abs(v[k]));
    #pragma unroll
    for (int d = 1; d < 8; d <<= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, d));
    const uint32_t byte = scale_byte(a, FMT == LGN_E4M3 ? 8 : 15);
    const float inv = inverse_scale(byte);
    if (c0 < ldq) {
        uint4 q;
        q.x = code_quad<FMT>(v, inv); q.y = code_quad<FMT>(v + 4, inv);
        q.z = code_quad<FMT>(v + 8, inv); q.w = code_quad<FMT>(v + 12, inv);
        *reinterpret_cast<uint4 *>(codes + (uint64_t)row * ldq + c0) = q;
    }
    uint32_t word = byte << (8 * (lane >> 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    word |= __shfl_xor_sync(0xffffffffu, word, 16);
    if (lane == 0) scales[fp8_scale_word(row, grp, groups)] = word;
}

// ------------------------------------------------------------------ 128 x 128 tiles
// Transposed copies and square blocks.  A CTA keeps its tile in registers (thread: 8 consecutive
// rows x 8 consecutive columns), so the tile is read once for both copies.  Transposed codes go
// through shared memory as units of 8 bytes (8 rows of one column); unit u of column c sits at
// place u ^ (c / 8), which spreads the 16 lanes that write units of columns 8 apart over all banks.
template <int DT, int FMT, bool SQUARE, bool VEC>
__global__ void __launch_bounds__(256)
fp8_tile_kernel(const char *__restrict__ x, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t col_tiles,
                uint8_t *__restrict__ codes, uint32_t ldq, uint8_t *__restrict__ scales, uint32_t groups,
                uint8_t *__restrict__ codes_t, uint32_t ldq_t, uint8_t *__restrict__ scales_t, uint32_t groups_t) {
    __shared__ uint32_t col_max[128];
    __shared__ uint32_t all_max;
    __shared__ __align__(16) uint2 tr[128 * 16];
    dep_launch();
    if (threadIdx.x < 128) col_max[threadIdx.x] = 0u;
    if (threadIdx.x == 0) all_max = 0u;
    dep_wait();
    constexpr int ES = DT == LGN_F32 ? 4 : 2;
    constexpr int kTop = FMT == LGN_E4M3 ? 8 : 15;
    const uint32_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
    const uint32_t cl = (threadIdx.x & 15) * 8, rl = (threadIdx.x >> 4) * 8;          // within the tile
    const uint32_t c0 = ct * 128 + cl, r0 = rt * 128 + rl;
    float v[8][8];
    const int valid = (int)min((int64_t)8, (int64_t)cols - (int64_t)c0);
    #pragma unroll
    for (int i = 0; i < 8; ++i)
        load_values<DT, 8, VEC>(x + ((uint64_t)(r0 + i) * ld + c0) * ES, r0 + i < rows ? valid : 0, v[i]);

    uint32_t rmax[8], cmax[8];
    #pragma unroll
    for (int j = 0; j < 8; ++j) cmax[j] = 0u;
    #pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t a = 0;
        #pragma unroll
        for (int j = 0; j < 8; ++j) { const uint32_t f = finite_abs(v[i][j]); a = max(a, f); cmax[j] = max(cmax[j], f); }
        rmax[i] = a;
    }
    __syncthreads();
    uint32_t row_byte[8], col_byte[8];
    if constexpr (SQUARE) {
        uint32_t a = 0;
        #pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, rmax[i]);
        a = __reduce_max_sync(0xffffffffu, a);
        if ((threadIdx.x & 31) == 0) atomicMax(&all_max, a);
        __syncthreads();
        const uint32_t b = scale_byte(all_max, kTop);
        #pragma unroll
        for (int i = 0; i < 8; ++i) row_byte[i] = col_byte[i] = b;
    } else {
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
            #pragma unroll
            for (int d = 1; d < 16; d <<= 1) rmax[i] = max(rmax[i], __shfl_xor_sync(0xffffffffu, rmax[i], d));
            row_byte[i] = scale_byte(rmax[i], kTop);
        }
        if (codes_t != nullptr) {
            #pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t a = max(cmax[j], __shfl_xor_sync(0xffffffffu, cmax[j], 16));
                if ((threadIdx.x & 16) == 0) atomicMax(&col_max[cl + j], a);
            }
            __syncthreads();
            #pragma unroll
            for (int j = 0; j < 8; ++j) col_byte[j] = scale_byte(col_max[cl + j], kTop);
        }
    }
    if (codes != nullptr) {
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float inv = inverse_scale(row_byte[i]);
            if (r0 + i < rows && c0 < ldq)                                            // ldq is a multiple of 16
                *reinterpret_cast<uint2 *>(codes + (uint64_t)(r0 + i) * ldq + c0) =
                    make_uint2(code_quad<FMT>(v[i], inv), code_quad<FMT>(v[i] + 4, inv));
            if ((threadIdx.x & 15) == 0)
                scales[4 * (uint64_t)fp8_scale_word(r0 + i, ct >> 2, groups) + (ct & 3)] = (uint8_t)row_byte[i];
        }
    }
    if (codes_t != nullptr) {
        #pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float inv = inverse_scale(col_byte[j]);
            float t[8];
            #pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = v[i][j];
            tr[(cl + j) * 16 + ((threadIdx.x >> 4) ^ (threadIdx.x & 15))] = make_uint2(code_quad<FMT>(t, inv), code_quad<FMT>(t + 4, inv));
            if (rl == 0) scales_t[4 * (uint64_t)fp8_scale_word(c0 + j, rt >> 2, groups_t) + (rt & 3)] = (uint8_t)col_byte[j];
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
#define LGN_TILE4(D, F) {{LGN_TILE(D, F, false, false), LGN_TILE(D, F, false, true)}, {LGN_TILE(D, F, true, false), LGN_TILE(D, F, true, true)}}
static const void *const kTileTable[2][2][2][2] = {{LGN_TILE4(LGN_F32, LGN_E4M3), LGN_TILE4(LGN_F32, LGN_E5M2)},
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
    const uint64_t es = dt == LGN_F32 ? 4 : 2, xb = ((rows - 1) * ld + cols) * es;
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
    return launch_dependent(kTileTable[dt][fmt][block == LGN_BLOCK_SQUARE][vec], dim3((unsigned)tiles), dim3(256), args, 0, stream);
}
