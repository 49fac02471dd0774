// Embedding lookup with scaling, and the gradient of the table.
//
//   out[t, :]    = scale * table[id_t, :]                       (zeros for an id outside the table)
//   dtable[v, :] (+)= scale * sum over { t : id_t = v } of dout[t, :]
//
// Both are bound by memory.  The gradient adds rows that share an id in a fixed order, without atomics on
// values: the tokens are sorted by id (stable), so that every table row owns one run of the sorted list.
//   sort_kernel    one cluster of 16 CTAs (8 where 16 do not fit): radix sort of (id, position), up to 9 bits per pass; on the way it marks the rows
//                  of the table that have a token (the marks are cleared by a memset before)
//   window_kernel  a warp per window of the sorted list and slab of columns walks its tokens, eight rows of dout in flight
//                  whatever the runs' lengths, and writes each run that lies inside the window to its table row; the
//                  pieces of runs that reach beyond it (one at its start, one at its end) go to scratch.  CTAs of the
//                  same launch, mixed in between, write zeros to the rows without a token: most of the bytes that the
//                  gradient of a large table has to write, streamed beside the gathers
//   join_kernel    adds the pieces of each run of several windows: a CTA per run and slab, its 8 warps a share of the pieces each
// so that no warp adds more than one window of tokens, or one window count of pieces, in sequence.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <mutex>

#include "lgn.h"
#include "lgn_launch.h"
#include "lgn_log.h"

namespace lgn {

constexpr uint64_t kEmbMaxTokens = 1ull << 30, kEmbMaxRows = (1ull << 31) - 2, kEmbMaxDim = 1ull << 24;

// ------------------------------------------------------------------ vectors of VE elements as fp32
template <int DT, int VE>
__device__ __forceinline__ void load_vec(const void *base, uint64_t i, float *v) {
    if constexpr (DT == LGN_F32) {
        const float *p = static_cast<const float *>(base) + i;
        if constexpr (VE == 8) {
            #pragma unroll
            for (int k = 0; k < 8; k += 4)
                asm volatile("ld.global.nc.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[k]), "=f"(v[k + 1]), "=f"(v[k + 2]), "=f"(v[k + 3]) : "l"(p + k));
        } else if constexpr (VE == 2) {
            const uint64_t w = ldro_u64(p);
            v[0] = __uint_as_float((uint32_t)w); v[1] = __uint_as_float((uint32_t)(w >> 32));
        } else v[0] = __uint_as_float(ldro_u32(p));
    } else {
        const unsigned short *p = static_cast<const unsigned short *>(base) + i;
        if constexpr (VE == 8) {
            uint32_t w[4];
            asm volatile("ld.global.nc.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
            #pragma unroll
            for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
        } else if constexpr (VE == 2) {
            const uint32_t w = ldro_u32(p);
            v[0] = __uint_as_float(w << 16); v[1] = __uint_as_float(w & 0xffff0000u);
        } else v[0] = __uint_as_float(ldro_u16(p) << 16);
    }
}

template <int DT, int VE>
__device__ __forceinline__ void load_vec_rw(const void *base, uint64_t i, float *v) {      // memory this kernel or the one before wrote
    if constexpr (VE == 8 && DT == LGN_F32) {
        const float4 a = reinterpret_cast<const float4 *>(static_cast<const float *>(base) + i)[0], b = reinterpret_cast<const float4 *>(static_cast<const float *>(base) + i)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else if constexpr (VE == 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(static_cast<const unsigned short *>(base) + i);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
        #pragma unroll
        for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
    } else {
        #pragma unroll
        for (int k = 0; k < VE; ++k) {
            if constexpr (DT == LGN_F32) v[k] = static_cast<const float *>(base)[i + k];
            else v[k] = __bfloat162float(static_cast<const __nv_bfloat16 *>(base)[i + k]);
        }
    }
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

template <int DT, int VE>
__device__ __forceinline__ void store_vec(void *base, uint64_t i, const float *v) {
    if constexpr (DT == LGN_F32) {
        float *p = static_cast<float *>(base) + i;
        if constexpr (VE == 8) {
            __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
            __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
        } else if constexpr (VE == 2) __stcs(reinterpret_cast<float2 *>(p), make_float2(v[0], v[1]));
        else __stcs(p, v[0]);
    } else {
        __nv_bfloat16 *p = static_cast<__nv_bfloat16 *>(base) + i;
        if constexpr (VE == 8)
            __stcs(reinterpret_cast<uint4 *>(p), make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])));
        else if constexpr (VE == 2) __stcs(reinterpret_cast<uint32_t *>(p), bf16_pair(v[0], v[1]));
        else *p = __float2bfloat16_rn(v[0]);
    }
}

// A vector as it lies in memory, for loads that are in flight together.
template <int DT, int VE> struct RawVec {
    static constexpr int kWords = VE * (DT == LGN_F32 ? 4 : 2) / 4 > 0 ? VE * (DT == LGN_F32 ? 4 : 2) / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void *base, uint64_t i) {
        const char *p = static_cast<const char *>(base) + i * (DT == LGN_F32 ? 4 : 2);
        if constexpr (kWords >= 4) {
            #pragma unroll
            for (int k = 0; k < kWords; k += 4)
                asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3]) : "l"(p + 4 * k));
        } else if constexpr (kWords == 2) asm volatile("ld.global.nc.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
        else if constexpr (DT == LGN_BF16 && VE == 1) w[0] = ldro_u16(p);
        else w[0] = ldro_u32(p);
    }
    __device__ __forceinline__ float at(int k) const {
        if constexpr (DT == LGN_F32) return __uint_as_float(w[k]);
        else return k & 1 ? __uint_as_float(w[k >> 1] & 0xffff0000u) : __uint_as_float(w[k >> 1] << 16);
    }
};

__device__ __forceinline__ int64_t load_id(const void *ids, uint64_t i, uint32_t wide) {
    return wide ? (int64_t)ldro_u64(static_cast<const int64_t *>(ids) + i) : (int64_t)(int32_t)ldro_u32(static_cast<const int32_t *>(ids) + i);
}

// ------------------------------------------------------------------ lookup
// Three mappings.  Rows of whole 16-byte pieces (lookup_kernel): items of 8 columns of one token, numbered along the output; a
// thread takes four, 256 apart, so that all threads work whatever the row's length and four rows' loads are in flight.
// Other rows (lookup_rows_kernel): 2^span_log2 threads walk a row, one or two elements at a time; a division per element
// would cost more than the idle threads (65536 x 999 bf16: 181 us against 94; sixteen narrow loads in flight instead of
// four: 136).
template <int TDT, int ODT, int VE>
__global__ void __launch_bounds__(256)
lookup_kernel(const void *table, uint64_t ld_table, uint64_t vocab, uint32_t chunks, const void *ids, uint32_t wide,
              uint64_t tokens, float scale, void *out, uint64_t ld_out, unsigned long long *outside) {
    dep_launch();
    const uint64_t start = (uint64_t)blockIdx.x * 1024, t0 = start / chunks;
    const uint32_t rest = (uint32_t)(start - t0 * chunks);
    uint64_t t[4];
    uint32_t c[4];
    int64_t id[4];
    dep_wait();
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t i = rest + k * 256 + threadIdx.x, q = i / chunks;
        t[k] = t0 + q;
        c[k] = (i - q * chunks) * VE;
        id[k] = t[k] < tokens ? load_id(ids, t[k], wide) : 0;
    }
    float v[4][VE];
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (id[k] < 0 || (uint64_t)id[k] >= vocab) {
            id[k] = -1;
            if (outside != nullptr && c[k] == 0 && t[k] < tokens) atomicAdd(outside, 1ull);
        }
        #pragma unroll
        for (int j = 0; j < VE; ++j) v[k][j] = 0.0f;
        if (id[k] >= 0 && t[k] < tokens) load_vec<TDT, VE>(table, (uint64_t)id[k] * ld_table + c[k], v[k]);
    }
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (t[k] >= tokens) break;
        if (id[k] >= 0 && scale != 1.0f) {
            #pragma unroll
            for (int j = 0; j < VE; ++j) v[k][j] *= scale;
        }
        store_vec<ODT, VE>(out, t[k] * ld_out + c[k], v[k]);
    }
}

template <int TDT, int ODT, int VE>
__global__ void __launch_bounds__(256)
lookup_rows_kernel(const void *table, uint64_t ld_table, uint64_t vocab, uint32_t chunks, const void *ids, uint32_t wide,
                   uint64_t tokens, float scale, void *out, uint64_t ld_out, unsigned long long *outside, uint32_t span_log2) {
    dep_launch();
    const uint32_t span = 1u << span_log2, rows = 256u >> span_log2, x = threadIdx.x & (span - 1);
    const uint64_t t0 = (uint64_t)blockIdx.x * (4 * rows) + (threadIdx.x >> span_log2);
    int64_t id[4];
    dep_wait();
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t t = t0 + k * rows;
        id[k] = t < tokens ? load_id(ids, t, wide) : 0;
        if (id[k] < 0 || (uint64_t)id[k] >= vocab) {
            id[k] = -1;
            if (outside != nullptr && x == 0 && t < tokens) atomicAdd(outside, 1ull);
        }
    }
    for (uint32_t c = x; c < chunks; c += span) {
        float v[4][VE];
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            #pragma unroll
            for (int j = 0; j < VE; ++j) v[k][j] = 0.0f;
            if (id[k] >= 0 && t0 + k * rows < tokens) load_vec<TDT, VE>(table, (uint64_t)id[k] * ld_table + (uint64_t)c * VE, v[k]);
        }
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (t0 + k * rows >= tokens) break;
            if (id[k] >= 0 && scale != 1.0f) {
                #pragma unroll
                for (int j = 0; j < VE; ++j) v[k][j] *= scale;
            }
            store_vec<ODT, VE>(out, (t0 + k * rows) * ld_out + (uint64_t)c * VE, v[k]);
        }
    }
}

// The third mapping, for a bf16 output without gaps whose rows are not whole 16-byte pieces: items are the 16-byte pieces of
// the output's memory, each of them part of one row or of two, filled by element loads (neighbours share their lines
// in L1) and stored at once instead of two bytes at a time (65536 x 999: 93 -> 78 us; with an fp32 output, whose
// elements are stored four bytes at a time, 21547 x 679 went from 21 to 24 us).  dim >= 8.
template <int TDT>
__global__ void __launch_bounds__(256)
lookup_flat_kernel(const void *table, uint64_t ld_table, uint64_t vocab, uint32_t dim, const void *ids, uint32_t wide,
                   uint64_t tokens, float scale, void *out, unsigned long long *outside) {
    constexpr int kPer = 8;
    dep_launch();
    // elements between the 16-byte boundary at or below the output's first element and that element
    const uint32_t lead = (uint32_t)(reinterpret_cast<uintptr_t>(out) & 15) / (16 / kPer);
    const uint64_t total = tokens * dim, first = (uint64_t)blockIdx.x * (1024 * kPer);
    const uint64_t start = first < lead ? 0 : first - lead, t0 = start / dim;
    const uint32_t rest = (uint32_t)(start - t0 * dim);
    dep_wait();
    #pragma unroll
    for (int half = 0; half < 4; half += 2) {
        uint64_t e[2];
        float v[2][kPer];
        uint32_t from_table[2] = {0u, 0u};                 // a bit per element
        #pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t n = ((half + k) * 256 + threadIdx.x) * kPer, skip = first + n < lead ? lead - (uint32_t)(first + n) : 0;   // skip: only in the first piece
            const uint32_t i = rest + (first < lead ? (n < lead ? 0 : n - lead) : n), q = i / dim, c = i - q * dim;
            const uint64_t t = t0 + q;
            e[k] = first + n;                              // counted from the boundary
            int64_t id[2] = {-1, -1};
            if (t < tokens) id[0] = load_id(ids, t, wide);
            if (c + kPer > dim && t + 1 < tokens) id[1] = load_id(ids, t + 1, wide);
            const bool in0 = id[0] >= 0 && (uint64_t)id[0] < vocab, in1 = id[1] >= 0 && (uint64_t)id[1] < vocab;
            if (outside != nullptr) {                      // a token is counted by the piece that holds its first column
                if (c == 0 && t < tokens && !in0) atomicAdd(outside, 1ull);
                if (c + kPer - skip > dim && t + 1 < tokens && !in1) atomicAdd(outside, 1ull);
            }
            #pragma unroll
            for (int j = 0; j < kPer; ++j) {
                v[k][j] = 0.0f;
                const uint32_t x = c + j - skip;           // column, counted on into the next row
                if ((uint32_t)j >= skip && (x < dim ? in0 : in1)) {
                    load_vec<TDT, 1>(table, x < dim ? (uint64_t)id[0] * ld_table + x : (uint64_t)id[1] * ld_table + (x - dim), &v[k][j]);
                    from_table[k] |= 1u << j;
                }
            }
        }
        #pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (scale != 1.0f) {
                #pragma unroll
                for (int j = 0; j < kPer; ++j) if (from_table[k] >> j & 1) v[k][j] *= scale;
            }
            if (e[k] >= lead && e[k] + kPer <= total + lead) {
                reinterpret_cast<uint4 *>(static_cast<unsigned short *>(out) + (e[k] - lead))[0] =
                    make_uint4(bf16_pair(v[k][0], v[k][1]), bf16_pair(v[k][2], v[k][3]), bf16_pair(v[k][4], v[k][5]), bf16_pair(v[k][6], v[k][7]));
            } else {
                #pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (e[k] + j >= lead && e[k] + j < total + lead) store_vec<LGN_BF16, 1>(out, e[k] + j - lead, &v[k][j]);
            }
        }
    }
}

// ------------------------------------------------------------------ sort
constexpr int kSortThreads = 1024, kSortBins = 512;
constexpr int kSortBatch = 8;                              // loads a lane has in flight
constexpr uint64_t kSortAlone = 1024;                      // tokens that one CTA sorts by itself (4999: 24 us, 16 with a cluster)

__device__ __forceinline__ uint64_t ld_l2(const uint64_t *p) {       // written by other CTAs of the cluster before its barrier
    uint64_t v;
    asm volatile("ld.global.cg.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ void cluster_sync_all() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct SortArgs {
    const void *ids;
    uint64_t *pair[2];             // id << 32 | position
    uint8_t *present;              // per table row: has a token (not used when the gradient is accumulated)
    uint64_t vocab;
    int64_t padding;
    uint32_t tokens, wide, bits, passes;
};

__device__ __forceinline__ uint32_t key_of(const SortArgs &a, uint32_t i) {       // vocab: left out, sorts last
    const int64_t id = load_id(a.ids, i, a.wide);
    return id < 0 || (uint64_t)id >= a.vocab || id == a.padding ? (uint32_t)a.vocab : (uint32_t)id;
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_kernel(const SortArgs a) {
    extern __shared__ uint32_t hist[];                     // [32][bins]
    __shared__ uint32_t total[kSortBins], base[kSortBins], warp_sum[32];
    dep_launch();
    dep_wait();
    uint32_t rank, ctas;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1u << a.bits, mask = bins - 1;
    const uint32_t per = (((a.tokens + ctas * 32 - 1) / (ctas * 32)) + 31u) & ~31u;
    const uint64_t lo64 = (uint64_t)(rank * 32 + warp) * per;
    const uint32_t lo = lo64 < a.tokens ? (uint32_t)lo64 : a.tokens, hi = lo64 + per < a.tokens ? (uint32_t)(lo64 + per) : a.tokens;
    for (uint32_t pass = 0; pass < a.passes; ++pass) {
        const uint64_t *src = a.pair[(pass + 1) & 1];
        uint64_t *dst = a.pair[pass & 1];
        const uint32_t shift = pass * a.bits;
        auto pair_at = [&](uint32_t i) -> uint64_t { return pass > 0 ? ld_l2(src + i) : (uint64_t)key_of(a, i) << 32 | i; };
        for (uint32_t i = threadIdx.x; i < 32 * bins; i += kSortThreads) hist[i] = 0u;
        __syncthreads();
        uint32_t *mine = hist + warp * bins;
        const bool once = per <= 32 * kSortBatch;              // a warp's share stays in registers from the count to the scatter
        uint64_t kb[kSortBatch];
        for (uint32_t i = lo + lane; i - lane < hi; i += 32 * kSortBatch) {
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j) kb[j] = i + 32 * j < hi ? pair_at(i + 32 * j) : 0u;
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j)
                if (i + 32 * j < hi) {
                    const uint32_t k = (uint32_t)(kb[j] >> 32);
                    atomicAdd(mine + ((k >> shift) & mask), 1u);
                    if (pass == 0 && a.present != nullptr && k < a.vocab) a.present[k] = 1;
                }
        }
        __syncthreads();
        if (threadIdx.x < bins) {                          // places of each warp within its CTA, digit by digit
            uint32_t run = 0;
            #pragma unroll 8
            for (int w = 0; w < 32; ++w) { const uint32_t c = hist[w * bins + threadIdx.x]; hist[w * bins + threadIdx.x] = run; run += c; }
            total[threadIdx.x] = run;
        }
        cluster_sync_all();
        uint32_t before = 0, all = 0;
        if (threadIdx.x < bins) {
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(total + threadIdx.x);
            #pragma unroll 8
            for (uint32_t c = 0; c < ctas; ++c) {
                uint32_t remote, v;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(c));
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
                if (c < rank) before += v;
                all += v;
            }
        }
        uint32_t inc = all;                                // exclusive sum over the digits (bins <= 512: warps 0..15)
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) { const uint32_t o = __shfl_up_sync(0xffffffffu, inc, d); if (lane >= d) inc += o; }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        if (threadIdx.x < bins) {
            uint32_t w0 = 0;
            for (uint32_t w = 0; w < warp; ++w) w0 += warp_sum[w];
            base[threadIdx.x] = w0 + inc - all + before;
        }
        __syncthreads();
        for (uint32_t i0 = lo + lane; i0 - lane < hi; i0 += 32 * kSortBatch) {
            if (!once) {
                #pragma unroll
                for (int j = 0; j < kSortBatch; ++j) kb[j] = i0 + 32 * j < hi ? pair_at(i0 + 32 * j) : 0u;
            }
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                if (i0 - lane + 32 * j >= hi) break;
                const bool on = i0 + 32 * j < hi;
                const uint32_t digit = on ? (uint32_t)(kb[j] >> (32 + shift)) & mask : bins;         // lanes past the end: a digit of their own
                const uint32_t same = __match_any_sync(0xffffffffu, digit);
                uint32_t at = 0;
                if (on) at = mine[digit];
                __syncwarp();
                if (on) {
                    const uint32_t r = __popc(same & ((1u << lane) - 1u));
                    if (r == 0) mine[digit] = at + __popc(same);
                    at += base[digit] + r;
                    dst[at] = kb[j];
                }
                __syncwarp();
            }
        }
        cluster_sync_all();
    }
}

// ------------------------------------------------------------------ sums
// The id of sorted place i.
__device__ __forceinline__ uint32_t id_at(const uint64_t *pair, uint64_t i) { return reinterpret_cast<const uint32_t *>(pair + i)[1]; }

struct SumArgs {
    const void *dout;
    uint64_t ld_dout;
    const uint64_t *pair;
    float *part;                   // two rows of `pitch` values per window: the piece at its start, the piece at its end
    uint32_t *long_count, *long_runs;   // windows with a run that begins there and reaches beyond: how many, and which
    void *out;
    uint64_t ld_out, vocab;
    uint32_t tokens, window_log2, windows, dim, pitch, slabs, accumulate;
    float scale;
    const uint8_t *present;        // as in SortArgs
    uint64_t ld_out_bytes, dim_bytes;
    uint32_t zero_unit, zero_blocks;   // table rows per CTA that writes zeros, and the number of those CTAs
};

// Zeros to the rows [first, last) without a token.  Rows of 1 KiB and more: a warp per row.  Shorter rows that follow one
// another without gaps are taken as one stretch of memory, 16 bytes per thread and step whatever the rows' length (91 bf16
// columns: 100 -> 26 us a call; 278 columns: 39 -> 32; 502 fp32 columns: 42 -> 57, hence the limit); a piece that also holds
// part of a row with a token is written in two-byte steps.
constexpr uint32_t kFlatRowBytes = 1024;
__device__ __forceinline__ void zero_rows(const SumArgs &a, uint64_t first, uint64_t last) {
    char *out = static_cast<char *>(a.out) + first * a.ld_out_bytes;
    const uint8_t *present = a.present + first;
    const uint32_t rows = (uint32_t)(last - first);
    if (a.ld_out_bytes != a.dim_bytes || a.dim_bytes >= kFlatRowBytes || rows * a.dim_bytes * a.dim_bytes >= (1ull << 32)) {
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        // row r of a group of 256 is warp (r mod 8)'s, so that all warps of the CTA have rows of each group
        for (uint32_t r0 = 0; r0 < rows; r0 += 256) {
            uint8_t mark = 1;
            const uint32_t mine = r0 + 8 * lane + warp;
            if (mine < rows) mark = present[mine];
            uint32_t todo = __ballot_sync(0xffffffffu, mark == 0);
            while (todo != 0) {
                const uint32_t k = __ffs(todo) - 1;
                todo &= todo - 1;
                char *row = out + (uint64_t)(r0 + 8 * k + warp) * a.ld_out_bytes, *end = row + a.dim_bytes;
                char *body = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(row) + 15) & ~(uintptr_t)15);
                if (body > end) body = end;
                const uint64_t vec = (uint64_t)(end - body) / 16;
                for (char *q = row + 2 * lane; q < body; q += 64) *reinterpret_cast<uint16_t *>(q) = 0;      // at most 14 bytes
                for (uint64_t v = lane; v < vec; v += 32) __stcs(reinterpret_cast<uint4 *>(body) + v, make_uint4(0, 0, 0, 0));
                for (char *q = body + vec * 16 + 2 * lane; q < end; q += 64) *reinterpret_cast<uint16_t *>(q) = 0;
            }
        }
        return;
    }
    // byte o of the stretch lies in row floor(o / d) = umulhi(o, ceil(2^32 / d)): exact while o d < 2^32
    const uint32_t d = (uint32_t)a.dim_bytes, bytes = rows * d, magic = 0xffffffffu / d + 1;
    const uint32_t lead = (uint32_t)(reinterpret_cast<uintptr_t>(out) & 15);        // pieces start at 16-byte boundaries
    for (uint32_t v = threadIdx.x; v * 16 < bytes + lead; v += 256) {
        const uint32_t lo = v == 0 ? 0 : v * 16 - lead, hi = min(v * 16 + 16 - lead, bytes);
        const uint32_t r0 = __umulhi(lo, magic), r1 = __umulhi(hi - 1, magic);
        bool all = hi - lo == 16;
        for (uint32_t r = r0; r <= r1; ++r) all = all && !present[r];
        if (all) { __stcs(reinterpret_cast<uint4 *>(out + lo), make_uint4(0, 0, 0, 0)); continue; }
        for (uint32_t q = lo; q < hi; q += 2)
            if (!present[__umulhi(q, magic)]) *reinterpret_cast<uint16_t *>(out + q) = 0;
    }
}

// The columns of a lane: 256 per warp, in 8 / VE vectors 32 VE apart, so that a row whose length or address allows
// no wide access still has 8 columns per lane to share the work per token.
template <int VE> struct Columns {
    static constexpr int kReps = 8 / VE;
    uint32_t c, dim;
    __device__ __forceinline__ Columns(uint32_t slab, uint32_t dim_) : c(slab * 256 + (threadIdx.x & 31) * VE), dim(dim_) {}
    __device__ __forceinline__ uint32_t at(int rep) const { return c + rep * 32 * VE; }
    __device__ __forceinline__ bool on(int rep) const { return at(rep) < dim; }
};

template <int ODT, int VE>
__device__ __forceinline__ void write_row(const SumArgs &a, uint32_t row, const Columns<VE> &col, float *sum) {
    #pragma unroll
    for (int r = 0; r < Columns<VE>::kReps; ++r) {
        if (!col.on(r)) continue;
        const uint64_t at = (uint64_t)row * a.ld_out + col.at(r);
        float *x = sum + r * VE;
        #pragma unroll
        for (int j = 0; j < VE; ++j) x[j] *= a.scale;
        if (a.accumulate) {
            float old[VE];
            load_vec_rw<ODT, VE>(a.out, at, old);
            #pragma unroll
            for (int j = 0; j < VE; ++j) x[j] += old[j];
        }
        store_vec<ODT, VE>(a.out, at, x);
    }
}

template <int DDT, int ODT, int VE>
__global__ void __launch_bounds__(256) window_kernel(const SumArgs a) {
    constexpr int kFlight = 8, kReps = Columns<VE>::kReps;
    dep_launch();
    dep_wait();
    // the CTAs that write zeros are spread evenly over the grid
    const uint64_t zb = (uint64_t)blockIdx.x * a.zero_blocks / gridDim.x, zn = (uint64_t)(blockIdx.x + 1) * a.zero_blocks / gridDim.x;
    if (zn != zb) {
        const uint64_t first = zb * a.zero_unit;
        zero_rows(a, first, first + a.zero_unit < a.vocab ? first + a.zero_unit : a.vocab);
        return;
    }
    const uint64_t item = (blockIdx.x - zb) * 8 + (threadIdx.x >> 5);
    const uint32_t w = (uint32_t)(item / a.slabs), lane = threadIdx.x & 31;
    const Columns<VE> col((uint32_t)(item % a.slabs), a.dim);
    if (w >= a.windows) return;
    const uint32_t lo = w << a.window_log2, hi = min(a.tokens, (w + 1) << a.window_log2);
    const uint32_t before = lo > 0 ? id_at(a.pair, lo - 1) : 0xffffffffu, after = hi < a.tokens ? id_at(a.pair, hi) : 0xffffffffu;
    float sum[8];
    uint32_t run = 0xffffffffu, first = id_at(a.pair, lo);
    auto flush = [&](uint32_t next) {                      // the run ends, or (next == run) goes on in the next window
        const bool from_before = run == first && before == run;
        if (!from_before && next != run) { write_row<ODT, VE>(a, run, col, sum); return; }
        if (!from_before && col.c == 0) a.long_runs[atomicAdd(a.long_count, 1u)] = w;    // once per window; the list's order is of no account
        float *q = a.part + (uint64_t)(2 * w + (from_before ? 0 : 1)) * a.pitch;
        #pragma unroll
        for (int r = 0; r < kReps; ++r) {
            if (!col.on(r)) continue;
            if constexpr (VE == 8) {
                reinterpret_cast<float4 *>(q + col.at(r))[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
                reinterpret_cast<float4 *>(q + col.at(r))[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
            } else {
                #pragma unroll
                for (int j = 0; j < VE; ++j) q[col.at(r) + j] = sum[r * VE + j];
            }
        }
    };
    for (uint32_t i0 = lo; i0 < hi; i0 += 32) {
        const uint32_t m = min(32u, hi - i0);
        const uint64_t mine = lane < m ? a.pair[i0 + lane] : a.vocab << 32;
        const uint32_t keys = (uint32_t)(mine >> 32), poss = (uint32_t)mine;
        for (uint32_t k0 = 0; k0 < m; k0 += kFlight) {
            if (__shfl_sync(0xffffffffu, keys, k0) >= a.vocab) { i0 = hi; break; }      // only left-out tokens follow
            RawVec<DDT, VE> v[kFlight][kReps];
            #pragma unroll
            for (int k = 0; k < kFlight; ++k) {
                const uint32_t p = __shfl_sync(0xffffffffu, poss, k0 + k), key = __shfl_sync(0xffffffffu, keys, k0 + k);
                #pragma unroll
                for (int r = 0; r < kReps; ++r)
                    if (key < a.vocab && col.on(r)) v[k][r].load(a.dout, (uint64_t)p * a.ld_dout + col.at(r));
            }
            #pragma unroll
            for (int k = 0; k < kFlight; ++k) {
                const uint32_t key = __shfl_sync(0xffffffffu, keys, k0 + k);
                if (key >= a.vocab) break;
                const bool fresh = key != run;
                if (fresh) {
                    if (run != 0xffffffffu) flush(key);
                    run = key;
                }
                #pragma unroll
                for (int r = 0; r < kReps; ++r) {
                    #pragma unroll
                    for (int j = 0; j < VE; ++j) sum[r * VE + j] = fresh ? v[k][r].at(j) : sum[r * VE + j] + v[k][r].at(j);
                }
            }
        }
    }
    if (run != 0xffffffffu) flush(after);
}

// Runs that begin in one window and reach beyond it.
template <int ODT, int VE>
__global__ void __launch_bounds__(256) join_kernel(const SumArgs a) {
    constexpr int kReps = Columns<VE>::kReps;
    __shared__ float sh[7][256];
    dep_launch();
    dep_wait();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t items = (uint64_t)*a.long_count * a.slabs;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t w = a.long_runs[item / a.slabs];
        const Columns<VE> col((uint32_t)(item % a.slabs), a.dim);
        const uint32_t run = id_at(a.pair, ((uint64_t)(w + 1) << a.window_log2) - 1);
        uint32_t end = w + 1;                              // one past the last window whose first token is of this run
        for (;;) {
            const uint32_t q = end + lane;
            const bool mine = q < a.windows && id_at(a.pair, (uint64_t)q << a.window_log2) == run;
            const uint32_t not_mine = __ballot_sync(0xffffffffu, !mine);
            if (not_mine != 0) { end += __ffs(not_mine) - 1; break; }
            end += 32;
        }
        // pieces: the end of window w, then the starts of windows w + 1 .. end - 1; warp q adds its share of them in order
        float sum[8];
        #pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        auto piece = [&](uint32_t i, float *x) {           // piece i: row 2 w + 1, then 2 (w + i)
            const uint64_t row = i == 0 ? 2 * (uint64_t)w + 1 : 2 * (uint64_t)(w + i);
            #pragma unroll
            for (int r = 0; r < kReps; ++r)
                if (col.on(r)) load_vec_rw<LGN_F32, VE>(a.part, row * a.pitch + col.at(r), x + r * VE);
        };
        const uint32_t pieces = end - w, per = (pieces + 7) / 8, i0 = min(pieces, warp * per), i1 = min(pieces, i0 + per);
        for (uint32_t i = i0; i < i1; i += 4) {
            float v[4][8];
            #pragma unroll
            for (int k = 0; k < 4; ++k) {
                #pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] = 0.0f;
                if (i + k < i1) piece(i + k, v[k]);
            }
            #pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < i1) {
                    #pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += v[k][j];
                }
        }
        if (warp > 0) {
            #pragma unroll
            for (int j = 0; j < 8; ++j) sh[warp - 1][j * 32 + lane] = sum[j];
        }
        __syncthreads();
        if (warp == 0) {
            #pragma unroll
            for (int q = 0; q < 7; ++q) {
                #pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += sh[q][j * 32 + lane];
            }
            write_row<ODT, VE>(a, run, col, sum);
        }
        __syncthreads();
    }
}

// Tokens per window: 8 (a batch of loads) to about a quarter of the square root of the tokens, the longer ones only where
// that leaves 16 warps per SM: a warp walks its window alone (1022 tokens x 2402: 35 us with 32, see join_kernel for what
// short windows leave to add).
static uint32_t window_log2_for(uint64_t tokens, uint64_t slabs) {
    uint32_t l = 3;
    while (l < 20 && (1ull << (2 * l + 4)) < tokens && (tokens * slabs >> (l + 1)) >= 2368) ++l;
    return l;
}

struct GradLayout { size_t long_runs, present, list, pair[2], part, total; uint32_t window_log2, windows, pitch; };

static bool grad_layout(uint64_t tokens, uint64_t vocab, uint64_t dim, GradLayout &l) {
    if (tokens > kEmbMaxTokens || vocab > kEmbMaxRows || dim > kEmbMaxDim) return false;
    l.window_log2 = window_log2_for(tokens, (dim + 255) / 256);
    l.windows = (uint32_t)((tokens + (1ull << l.window_log2) - 1) >> l.window_log2);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~(size_t)255; return here; };
    l.long_runs = take(256 + vocab);                       // the list's count and, 256 bytes on, the marks: cleared by one memset
    l.present = l.long_runs + 256;
    l.list = take((size_t)l.windows * 4);
    for (int i = 0; i < 2; ++i) l.pair[i] = take(tokens * 8);
    l.pitch = (uint32_t)((dim + 7) & ~7ull);
    l.part = take(l.windows > 1 ? (size_t)2 * l.windows * l.pitch * 4 : 0);
    l.total = at < 256 ? 256 : at;
    return true;
}

// CTAs of the sort's cluster on the current device: 16 where the device can place such a cluster, else 8.  Found once per device;
// 0: the runtime refused.
static int sort_ctas() {
    static std::mutex guard;
    static int found[64];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
    std::lock_guard<std::mutex> lock(guard);
    if (dev < 64 && found[dev] != 0) return found[dev];
    const void *fn = reinterpret_cast<const void *>(&sort_kernel);
    const int smem = 32 * kSortBins * 4;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { (void)cudaGetLastError(); return 0; }
    int n = 8;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 16;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.gridDim = dim3(16);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = (size_t)smem;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, fn, &cfg) == cudaSuccess && clusters >= 1) n = 16;
    }
    (void)cudaGetLastError();
    if (dev < 64) found[dev] = n;
    return n;
}

// Elements per access: 8 where every row of both matrices starts at a multiple of 16 bytes and holds
// a multiple of 8 elements, 2 likewise with pairs, else 1.
static int vector_of(uint64_t dim, const void *a, uint64_t lda, uint64_t ea, const void *b, uint64_t ldb, uint64_t eb) {
    if (dim % 8 == 0 && aligned_to(a, 16) && aligned_to(b, 16) && (lda * ea) % 16 == 0 && (ldb * eb) % 16 == 0) return 2;
    if (dim % 2 == 0 && aligned_to(a, 2 * ea) && aligned_to(b, 2 * eb) && lda % 2 == 0 && ldb % 2 == 0) return 1;
    return 0;
}

#define LGN_LK(T, O) {reinterpret_cast<const void *>(&lookup_rows_kernel<T, O, 1>), reinterpret_cast<const void *>(&lookup_rows_kernel<T, O, 2>), reinterpret_cast<const void *>(&lookup_kernel<T, O, 8>)}
static const void *const kLookupTable[2][2][3] = {{LGN_LK(LGN_F32, LGN_F32), LGN_LK(LGN_F32, LGN_BF16)}, {LGN_LK(LGN_BF16, LGN_F32), LGN_LK(LGN_BF16, LGN_BF16)}};
#undef LGN_LK
static const void *const kLookupFlatTable[2] = {reinterpret_cast<const void *>(&lookup_flat_kernel<LGN_F32>), reinterpret_cast<const void *>(&lookup_flat_kernel<LGN_BF16>)};
#define LGN_WK(T, O) {reinterpret_cast<const void *>(&window_kernel<T, O, 1>), reinterpret_cast<const void *>(&window_kernel<T, O, 2>), reinterpret_cast<const void *>(&window_kernel<T, O, 8>)}
static const void *const kWindowTable[2][2][3] = {{LGN_WK(LGN_F32, LGN_F32), LGN_WK(LGN_F32, LGN_BF16)}, {LGN_WK(LGN_BF16, LGN_F32), LGN_WK(LGN_BF16, LGN_BF16)}};
#undef LGN_WK
#define LGN_JK(O) {reinterpret_cast<const void *>(&join_kernel<O, 1>), reinterpret_cast<const void *>(&join_kernel<O, 2>), reinterpret_cast<const void *>(&join_kernel<O, 8>)}
static const void *const kJoinTable[2][3] = {LGN_JK(LGN_F32), LGN_JK(LGN_BF16)};
#undef LGN_JK
static const int kVe[3] = {1, 2, 8};

static uint64_t esize(lgn_dtype dt) { return dt == LGN_BF16 ? 2 : 4; }
static bool good_dtype(lgn_dtype dt) { return dt == LGN_F32 || dt == LGN_BF16; }

}  // namespace lgn

using namespace lgn;

extern "C" lgn_status lgn_embedding(const void *table, uint64_t vocab, uint64_t dim, uint64_t ld_table, lgn_dtype table_dt,
                                    const void *ids, int ids_bits, uint64_t tokens, double scale,
                                    void *out, uint64_t ld_out, lgn_dtype out_dt, uint64_t *n_outside_dev, void *stream) {
    if (!good_dtype(table_dt) || !good_dtype(out_dt) || (ids_bits != 32 && ids_bits != 64)) return LGN_ERR_INVALID_ARG;
    if (tokens > kEmbMaxTokens || vocab > kEmbMaxRows || dim > kEmbMaxDim) return LGN_ERR_UNSUPPORTED;
    if (!aligned_to(n_outside_dev, 8)) return LGN_ERR_INVALID_ARG;
    if (tokens == 0 || dim == 0) return LGN_OK;
    if (ld_table < dim || ld_out < dim || ld_table > (1ull << 30) || ld_out > (1ull << 30)) return LGN_ERR_INVALID_ARG;
    const uint64_t et = esize(table_dt), eo = esize(out_dt), ei = ids_bits / 8;
    if ((vocab > 0 && table == nullptr) || ids == nullptr || out == nullptr) return LGN_ERR_INVALID_ARG;
    if (!aligned_to(table, et) || !aligned_to(out, eo) || !aligned_to(ids, ei)) return LGN_ERR_INVALID_ARG;
    const uint64_t ob = ((tokens - 1) * ld_out + dim) * eo;
    if (ranges_overlap(out, ob, table, vocab ? ((vocab - 1) * ld_table + dim) * et : 0) || ranges_overlap(out, ob, ids, tokens * ei)) return LGN_ERR_INVALID_ARG;
    const int vi = vector_of(dim, table, ld_table, et, out, ld_out, eo);
    const uint64_t chunks = (dim + kVe[vi] - 1) / kVe[vi];
    if (kVe[vi] < 8 && dim >= 8 && ld_out == dim && out_dt == LGN_BF16) {
        const uint64_t pieces = (tokens * dim + 7) / 8 + 1, flat_blocks = (pieces + 1023) / 1024;
        if (flat_blocks > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
        uint32_t d = (uint32_t)dim, wide = ids_bits == 64;
        float s = (float)scale;
        unsigned long long *outside = reinterpret_cast<unsigned long long *>(n_outside_dev);
        log_line("embedding: %llu tokens, dim %u, pieces of the output, %llu CTAs", (unsigned long long)tokens, d, (unsigned long long)flat_blocks);
        void *args[] = {&table, &ld_table, &vocab, &d, &ids, &wide, &tokens, &s, &out, &outside};
        return launch_dependent(kLookupFlatTable[table_dt], dim3((unsigned)flat_blocks), dim3(256), args, 0, stream);
    }
    uint32_t span = 0;
    while (span < 8 && (1ull << span) < chunks) ++span;
    const uint64_t per = 4ull * (256u >> span), blocks = kVe[vi] == 8 ? (tokens * chunks + 1023) / 1024 : (tokens + per - 1) / per;
    if (blocks > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    uint32_t per_row = (uint32_t)chunks, wide = ids_bits == 64;
    float s = (float)scale;
    unsigned long long *outside = reinterpret_cast<unsigned long long *>(n_outside_dev);
    log_line("embedding: %llu tokens, dim %u, %d elements per access, %llu CTAs", (unsigned long long)tokens, (uint32_t)dim, kVe[vi], (unsigned long long)blocks);
    void *args[] = {&table, &ld_table, &vocab, &per_row, &ids, &wide, &tokens, &s, &out, &ld_out, &outside, &span};   // lookup_kernel takes no span
    return launch_dependent(kLookupTable[table_dt][out_dt][vi], dim3((unsigned)blocks), dim3(256), args, 0, stream);
}

extern "C" size_t lgn_embedding_grad_workspace_bytes(uint64_t tokens, uint64_t vocab, uint64_t dim) {
    GradLayout l;
    return grad_layout(tokens, vocab, dim, l) ? l.total : 0;
}

extern "C" lgn_status lgn_embedding_grad(const void *dout, uint64_t ld_dout, lgn_dtype dout_dt, const void *ids, int ids_bits, uint64_t tokens,
                                         uint64_t vocab, uint64_t dim, double scale, int64_t padding_idx,
                                         void *dtable, uint64_t ld_table, lgn_dtype table_dt, int accumulate,
                                         void *ws, size_t ws_bytes, void *stream) {
    if (!good_dtype(dout_dt) || !good_dtype(table_dt) || (ids_bits != 32 && ids_bits != 64)) return LGN_ERR_INVALID_ARG;
    GradLayout l;
    if (!grad_layout(tokens, vocab, dim, l)) return LGN_ERR_UNSUPPORTED;
    if (vocab == 0 || dim == 0) return LGN_OK;
    if (ld_dout < dim || ld_table < dim || ld_dout > (1ull << 30) || ld_table > (1ull << 30)) return LGN_ERR_INVALID_ARG;
    const uint64_t ed = esize(dout_dt), et = esize(table_dt), ei = ids_bits / 8;
    if ((tokens > 0 && (dout == nullptr || ids == nullptr)) || dtable == nullptr || ws == nullptr) return LGN_ERR_INVALID_ARG;
    if (!aligned_to(dout, ed) || !aligned_to(dtable, et) || !aligned_to(ids, ei) || !aligned_to(ws, 16)) return LGN_ERR_INVALID_ARG;
    if (ws_bytes < l.total) return LGN_ERR_WORKSPACE;
    const uint64_t db = tokens ? ((tokens - 1) * ld_dout + dim) * ed : 0, tb = ((vocab - 1) * ld_table + dim) * et;
    if (ranges_overlap(dtable, tb, dout, db) || ranges_overlap(dtable, tb, ids, tokens * ei) || ranges_overlap(ws, l.total, dout, db) ||
        ranges_overlap(ws, l.total, ids, tokens * ei) || ranges_overlap(ws, l.total, dtable, tb)) return LGN_ERR_INVALID_ARG;

    char *w = static_cast<char *>(ws);
    SortArgs s = {};
    s.ids = ids;
    for (int i = 0; i < 2; ++i) s.pair[i] = reinterpret_cast<uint64_t *>(w + l.pair[i]);
    s.present = reinterpret_cast<uint8_t *>(w + l.present);
   
    s.vocab = vocab;
    s.padding = padding_idx;
    s.tokens = (uint32_t)tokens;
    s.wide = ids_bits == 64;
    uint32_t bits = 1;
    while (bits < 32 && (vocab >> bits) != 0) ++bits;                 // keys 0 .. vocab
    s.passes = (bits + 8) / 9;
    s.bits = (bits + s.passes - 1) / s.passes;
    if (s.bits < 5) s.bits = 5;                                        // whole warps of digits
    const size_t smem = (size_t)32 * sizeof(uint32_t) << s.bits;
    const void *sort = reinterpret_cast<const void *>(&sort_kernel);
    const int most = sort_ctas();
    if (most == 0) return LGN_ERR_CUDA;
    // fewer CTAs have less to tell one another, more have shorter shares (whole call, 3000 / 8192 / 65536 tokens: 24.2 / 35.2 / 124 us with
    // 4 CTAs, 24.1 / 33.1 / 95 with 8, 26.0 / 33.6 / 86 with 16)
    const int ctas = tokens <= kSortAlone ? 1 : tokens <= 4096 ? 4 : tokens <= 8192 ? 8 : most;
    if (accumulate) {
        s.present = nullptr;
        if (tokens == 0) return LGN_OK;
    }
    if (cudaMemsetAsync(w + l.long_runs, 0, accumulate ? 256 : 256 + (size_t)vocab, static_cast<cudaStream_t>(stream)) != cudaSuccess) {
        (void)cudaGetLastError();
        return LGN_ERR_CUDA;
    }
    if (tokens > 0) {
        void *args[] = {&s};
        const lgn_status r = launch_dependent(sort, dim3((unsigned)ctas), dim3(kSortThreads), args, smem, stream, (unsigned)ctas);
        if (r != LGN_OK) return r;
    }
    const int vi = vector_of(dim, dout, ld_dout, ed, dtable, ld_table, et);
    SumArgs a = {};
    a.dout = dout; a.ld_dout = ld_dout;
    a.pair = s.pair[(s.passes + 1) & 1];
    a.part = reinterpret_cast<float *>(w + l.part);
    a.long_count = reinterpret_cast<uint32_t *>(w + l.long_runs);
    a.long_runs = reinterpret_cast<uint32_t *>(w + l.list);
    a.out = dtable; a.ld_out = ld_table; a.vocab = vocab;
    a.tokens = s.tokens;
    a.window_log2 = l.window_log2; a.windows = l.windows;
    a.dim = (uint32_t)dim; a.pitch = l.pitch;
    a.slabs = (uint32_t)((dim + 255) / 256);
    a.accumulate = accumulate != 0;
    a.scale = (float)scale;
    void *args[] = {&a};
    const uint64_t blocks = ((uint64_t)l.windows * a.slabs + 7) / 8;
    if (!accumulate) {
        // 8 to 256 KiB of the table a CTA, enough CTAs for every SM to have a few of them, at most 2^20 CTAs; at least 8 rows (a warp's each)
        const uint64_t row = dim * et, all = vocab * row / 1024;
        uint64_t unit = (all < (8u << 10) ? (8u << 10) : all > (256u << 10) ? (256u << 10) : all) / row;
        if (unit < 8) unit = 8;
        if (unit < (vocab >> 20) + 1) unit = (vocab >> 20) + 1;
        a.present = s.present;
        a.ld_out_bytes = ld_table * et; a.dim_bytes = row;
        a.zero_unit = (uint32_t)unit;
        a.zero_blocks = (uint32_t)((vocab + unit - 1) / unit);
    }
    if (blocks + a.zero_blocks > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    log_line("embedding_grad: %u tokens, %llu rows, dim %u, %u passes of %u bits, %u windows, %d elements per access", s.tokens,
             (unsigned long long)vocab, a.dim, s.passes, s.bits, l.windows, kVe[vi]);
    const lgn_status r = launch_dependent(kWindowTable[dout_dt][table_dt][vi], dim3((unsigned)blocks + a.zero_blocks), dim3(256), args, 0, stream);
    if (r != LGN_OK || l.windows <= 1) return r;
    const uint64_t runs = (uint64_t)(l.windows - 1) * a.slabs;            // no more runs than windows that have a successor
    return launch_dependent(kJoinTable[table_dt][vi], dim3((unsigned)(runs < 1184 ? runs : 1184)), dim3(256), args, 0, stream);
}
