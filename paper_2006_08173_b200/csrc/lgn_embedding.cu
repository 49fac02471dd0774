// Embedding lookup with scaling, and the gradient of the table.
//
//   out[t, :]    = scale * table[id_t, :]                       (zeros for an id outside the table)
//   dtable[v, :] (+)= scale * sum over { t : id_t = v } of dout[t, :]
//
// Both are bound by memory.  The gradient adds rows that share an id in a fixed order, without atomics on
// values: the tokens are sorted by id (stable), so that every table row owns one run of the sorted list.
//   sort_ids_kernel    one cluster of 8 CTAs: radix sort of (id, position), up to 9 bits per pass; then the
//                      first and last place of every id's run
//   window_kernel      runs longer than a window of the sorted list: the pieces a window holds of runs that
//                      reach beyond it are added up first, each by a warp of its own
//   rows_kernel        every row of the table: zeros, the sum of a run inside one window, or the sum of
//                      its windows' pieces
// so that no warp adds more than one window of tokens, or one window count of pieces, in sequence.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

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
__device__ __forceinline__ void load_vec_rw(const void *base, uint64_t i, float *v) {      // memory this kernel also writes
    #pragma unroll
    for (int k = 0; k < VE; ++k) {
        if constexpr (DT == LGN_F32) v[k] = static_cast<const float *>(base)[i + k];
        else v[k] = __bfloat162float(static_cast<const __nv_bfloat16 *>(base)[i + k]);
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

__device__ __forceinline__ int64_t load_id(const void *ids, uint64_t i, uint32_t wide) {
    return wide ? (int64_t)ldro_u64(static_cast<const int64_t *>(ids) + i) : (int64_t)(int32_t)ldro_u32(static_cast<const int32_t *>(ids) + i);
}

// ------------------------------------------------------------------ lookup
// A block takes 4 * (256 / span) tokens; `span` (a power of two) threads walk a row.
template <int TDT, int ODT, int VE>
__global__ void __launch_bounds__(256)
lookup_kernel(const void *__restrict__ table, uint64_t ld_table, uint64_t vocab, uint32_t dim, const void *__restrict__ ids, uint32_t wide,
              uint64_t tokens, float scale, void *__restrict__ out, uint64_t ld_out, uint32_t span_log2, unsigned long long *outside) {
    dep_launch();
    dep_wait();
    const uint32_t span = 1u << span_log2, rows = 256u >> span_log2, x = threadIdx.x & (span - 1);
    const uint64_t t0 = (uint64_t)blockIdx.x * (4 * rows) + (threadIdx.x >> span_log2);
    int64_t id[4];
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t t = t0 + k * rows;
        id[k] = t < tokens ? load_id(ids, t, wide) : 0;
        if (id[k] < 0 || (uint64_t)id[k] >= vocab) {
            id[k] = -1;
            if (outside != nullptr && x == 0 && t < tokens) atomicAdd(outside, 1ull);
        }
    }
    for (uint32_t c = x * VE; c < dim; c += span * VE) {
        float v[4][VE];
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            #pragma unroll
            for (int j = 0; j < VE; ++j) v[k][j] = 0.0f;
            if (id[k] >= 0 && t0 + k * rows < tokens) load_vec<TDT, VE>(table, (uint64_t)id[k] * ld_table + c, v[k]);
        }
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (t0 + k * rows >= tokens) break;
            if (id[k] >= 0 && scale != 1.0f) {
                #pragma unroll
                for (int j = 0; j < VE; ++j) v[k][j] *= scale;
            }
            store_vec<ODT, VE>(out, (t0 + k * rows) * ld_out + c, v[k]);
        }
    }
}

// ------------------------------------------------------------------ sort
constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortCtas * 32, kSortBins = 512;
constexpr int kSortBatch = 8;                              // loads a lane has in flight

__device__ __forceinline__ uint32_t ld_l2(const uint32_t *p) {       // written by other CTAs of the cluster before its barrier
    uint32_t v;
    asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ void cluster_sync_all() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct SortArgs {
    const void *ids;
    uint32_t *key[2], *pos[2];
    uint2 *run;                    // per table row: first and one past the last place in the sorted list
    uint64_t vocab;
    int64_t padding;
    uint32_t tokens, wide, bits, passes;
};

__global__ void __launch_bounds__(kSortThreads, 1) sort_ids_kernel(const SortArgs a) {
    extern __shared__ uint32_t hist[];                     // [32][kSortBins]
    __shared__ uint32_t total[kSortBins], base[kSortBins], warp_sum[32];
    dep_launch();
    dep_wait();
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1u << a.bits, mask = bins - 1;
    for (uint64_t i = rank * kSortThreads + threadIdx.x; i < a.vocab; i += kSortCtas * kSortThreads) a.run[i] = make_uint2(0u, 0u);
    const uint32_t per = (((a.tokens + kSortWarps - 1) / kSortWarps) + 31u) & ~31u;
    const uint64_t lo64 = (uint64_t)(rank * 32 + warp) * per;
    const uint32_t lo = lo64 < a.tokens ? (uint32_t)lo64 : a.tokens, hi = lo64 + per < a.tokens ? (uint32_t)(lo64 + per) : a.tokens;
    const uint32_t absent = (uint32_t)a.vocab;             // the key of tokens that are left out: sorts last
    for (uint32_t pass = 0; pass < a.passes; ++pass) {
        const uint32_t *ksrc = a.key[(pass + 1) & 1], *psrc = a.pos[(pass + 1) & 1];
        uint32_t *kdst = a.key[pass & 1], *pdst = a.pos[pass & 1];
        const uint32_t shift = pass * a.bits;
        auto key_at = [&](uint32_t i) -> uint32_t {
            if (pass > 0) return ld_l2(ksrc + i);
            const int64_t id = load_id(a.ids, i, a.wide);
            return id < 0 || (uint64_t)id >= a.vocab || id == a.padding ? absent : (uint32_t)id;
        };
        for (uint32_t i = threadIdx.x; i < 32 * bins; i += kSortThreads) hist[i] = 0u;
        __syncthreads();
        uint32_t *mine = hist + warp * bins;
        for (uint32_t i = lo + lane; i < hi; i += 32 * kSortBatch) {
            uint32_t k[kSortBatch];
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j) k[j] = i + 32 * j < hi ? key_at(i + 32 * j) : 0u;
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j) if (i + 32 * j < hi) atomicAdd(mine + ((k[j] >> shift) & mask), 1u);
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
            #pragma unroll
            for (uint32_t c = 0; c < kSortCtas; ++c) {
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
            uint32_t kb[kSortBatch], pb[kSortBatch];
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                const uint32_t i = i0 + 32 * j;
                kb[j] = i < hi ? key_at(i) : 0u;
                pb[j] = i < hi && pass > 0 ? ld_l2(psrc + i) : i;
            }
            #pragma unroll
            for (int j = 0; j < kSortBatch; ++j) {
                if (i0 - lane + 32 * j >= hi) break;
                const bool on = i0 + 32 * j < hi;
                const uint32_t digit = on ? (kb[j] >> shift) & mask : bins;         // lanes past the end: a digit of their own
                const uint32_t same = __match_any_sync(0xffffffffu, digit);
                uint32_t at = 0;
                if (on) at = mine[digit];
                __syncwarp();
                if (on) {
                    const uint32_t r = __popc(same & ((1u << lane) - 1u));
                    if (r == 0) mine[digit] = at + __popc(same);
                    at += base[digit] + r;
                    kdst[at] = kb[j];
                    pdst[at] = pb[j];
                }
                __syncwarp();
            }
        }
        cluster_sync_all();
    }
    const uint32_t *key = a.key[(a.passes + 1) & 1];
    for (uint32_t i = lo + lane; i < hi; i += 32) {
        const uint32_t k = ld_l2(key + i);
        if (k == absent) continue;
        if (i == 0 || ld_l2(key + i - 1) != k) a.run[k].x = i;
        if (i + 1 == a.tokens || ld_l2(key + i + 1) != k) a.run[k].y = i + 1;
    }
}

// ------------------------------------------------------------------ sums
// Adds dout rows pos[a..b) , columns c .. c + VE of each lane, in order.
template <int DDT, int VE>
__device__ __forceinline__ void add_rows(const void *dout, uint64_t ld, const uint32_t *pos, uint32_t a, uint32_t b, uint32_t c, bool on, float *sum) {
    const uint32_t lane = threadIdx.x & 31;
    #pragma unroll
    for (int j = 0; j < VE; ++j) sum[j] = 0.0f;
    for (uint32_t i0 = a; i0 < b; i0 += 32) {
        const uint32_t mine = i0 + lane < b ? ldro_u32(pos + i0 + lane) : 0u, m = min(32u, b - i0);
        for (uint32_t k0 = 0; k0 < m; k0 += 8) {
            float v[8][VE];
            #pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t p = __shfl_sync(0xffffffffu, mine, k0 + k);
                #pragma unroll
                for (int j = 0; j < VE; ++j) v[k][j] = 0.0f;
                if (on && k0 + k < m) load_vec<DDT, VE>(dout, (uint64_t)p * ld + c, v[k]);
            }
            #pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k0 + k < m) {
                    #pragma unroll
                    for (int j = 0; j < VE; ++j) sum[j] += v[k][j];
                }
        }
    }
}

struct SumArgs {
    const void *dout;
    uint64_t ld_dout;
    const uint32_t *key, *pos;
    const uint2 *run;
    float *part;                   // two rows of `pitch` values per window: the piece at its start, the piece at its end
    void *out;
    uint64_t ld_out, vocab;
    uint32_t tokens, window_log2, windows, dim, pitch, slabs, accumulate;
    float scale;
};

template <int DDT, int VE>
__global__ void __launch_bounds__(256) window_kernel(const SumArgs a) {
    dep_launch();
    dep_wait();
    const uint64_t item = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint32_t w = (uint32_t)(item / a.slabs), c = ((uint32_t)(item % a.slabs) * 32 + (threadIdx.x & 31)) * VE;
    if (w >= a.windows) return;
    const uint32_t lo = w << a.window_log2, hi = min(a.tokens, (w + 1) << a.window_log2);
    const bool on = c < a.dim;
    float sum[VE];
    auto put = [&](uint32_t row) {
        if (on) {
            #pragma unroll
            for (int j = 0; j < VE; ++j) a.part[(uint64_t)row * a.pitch + c + j] = sum[j];
        }
    };
    const uint32_t k0 = a.key[lo], k1 = a.key[hi - 1];
    if (k0 < a.vocab) {
        const uint2 r = a.run[k0];
        if (r.x < lo) { add_rows<DDT, VE>(a.dout, a.ld_dout, a.pos, lo, min(hi, r.y), c, on, sum); put(2 * w); }
    }
    if (k1 < a.vocab) {
        const uint2 r = a.run[k1];
        if (r.x >= lo && r.y > hi) { add_rows<DDT, VE>(a.dout, a.ld_dout, a.pos, r.x, hi, c, on, sum); put(2 * w + 1); }
    }
}

constexpr uint32_t kRowsPerWarp = 8;

template <int DDT, int ODT, int VE>
__global__ void __launch_bounds__(256) rows_kernel(const SumArgs a) {
    dep_launch();
    dep_wait();
    const uint64_t item = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint64_t v0 = item / a.slabs * kRowsPerWarp;
    const uint32_t lane = threadIdx.x & 31, c = ((uint32_t)(item % a.slabs) * 32 + lane) * VE;
    if (v0 >= a.vocab) return;
    const bool on = c < a.dim;
    const uint2 runs = lane < kRowsPerWarp && v0 + lane < a.vocab ? a.run[v0 + lane] : make_uint2(0u, 0u);
    for (uint32_t k = 0; k < kRowsPerWarp && v0 + k < a.vocab; ++k) {
        const uint32_t lo = __shfl_sync(0xffffffffu, runs.x, k), hi = __shfl_sync(0xffffffffu, runs.y, k);
        float sum[VE];
        const uint64_t at = (v0 + k) * a.ld_out + c;
        if (lo == hi) {
            if (!a.accumulate && on) {
                #pragma unroll
                for (int j = 0; j < VE; ++j) sum[j] = 0.0f;
                store_vec<ODT, VE>(a.out, at, sum);
            }
            continue;
        }
        const uint32_t w0 = lo >> a.window_log2, w1 = (hi - 1) >> a.window_log2;
        if (w0 == w1) add_rows<DDT, VE>(a.dout, a.ld_dout, a.pos, lo, hi, c, on, sum);
        else if (on) {
            // the piece of the first window is its end piece, unless the run covers that window from its start
            #pragma unroll
            for (int j = 0; j < VE; ++j) sum[j] = a.part[(uint64_t)(2 * w0 + 1) * a.pitch + c + j];
            #pragma unroll 8
            for (uint32_t w = w0 + 1; w <= w1; ++w) {
                #pragma unroll
                for (int j = 0; j < VE; ++j) sum[j] += a.part[(uint64_t)(2 * w) * a.pitch + c + j];
            }
        }
        if (on) {
            #pragma unroll
            for (int j = 0; j < VE; ++j) sum[j] *= a.scale;
            if (a.accumulate) {
                float old[VE];
                load_vec_rw<ODT, VE>(a.out, at, old);
                #pragma unroll
                for (int j = 0; j < VE; ++j) sum[j] += old[j];
            }
            store_vec<ODT, VE>(a.out, at, sum);
        }
    }
}

// Tokens per window: about a quarter of the square root of their number.  The square root itself would make the
// worst run (all tokens one id) shortest; real runs are far shorter, and short windows spread them over more warps.
static uint32_t window_log2_for(uint64_t tokens) {
    uint32_t l = 5;
    while (l < 20 && (1ull << (2 * l + 4)) < tokens) ++l;
    return l;
}

struct GradLayout { size_t run, key[2], pos[2], part, total; uint32_t window_log2, windows, pitch; };

static bool grad_layout(uint64_t tokens, uint64_t vocab, uint64_t dim, GradLayout &l) {
    if (tokens > kEmbMaxTokens || vocab > kEmbMaxRows || dim > kEmbMaxDim) return false;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~(size_t)255; return here; };
    l.run = take(vocab * 8);
    for (int i = 0; i < 2; ++i) { l.key[i] = take(tokens * 4); l.pos[i] = take(tokens * 4); }
    l.window_log2 = window_log2_for(tokens);
    l.windows = (uint32_t)((tokens + (1ull << l.window_log2) - 1) >> l.window_log2);
    l.pitch = (uint32_t)((dim + 7) & ~7ull);
    l.part = take(l.windows > 1 ? (size_t)2 * l.windows * l.pitch * 4 : 0);
    l.total = at < 256 ? 256 : at;
    return true;
}

// Elements per access: 8 where every row of both matrices starts at a multiple of 16 bytes and holds
// a multiple of 8 elements, 2 likewise with pairs, else 1.
static int vector_of(uint64_t dim, const void *a, uint64_t lda, uint64_t ea, const void *b, uint64_t ldb, uint64_t eb) {
    if (dim % 8 == 0 && aligned_to(a, 16) && aligned_to(b, 16) && (lda * ea) % 16 == 0 && (ldb * eb) % 16 == 0) return 2;
    if (dim % 2 == 0 && aligned_to(a, 2 * ea) && aligned_to(b, 2 * eb) && lda % 2 == 0 && ldb % 2 == 0) return 1;
    return 0;
}

#define LGN_LK(T, O) {reinterpret_cast<const void *>(&lookup_kernel<T, O, 1>), reinterpret_cast<const void *>(&lookup_kernel<T, O, 2>), reinterpret_cast<const void *>(&lookup_kernel<T, O, 8>)}
static const void *const kLookupTable[2][2][3] = {{LGN_LK(LGN_F32, LGN_F32), LGN_LK(LGN_F32, LGN_BF16)}, {LGN_LK(LGN_BF16, LGN_F32), LGN_LK(LGN_BF16, LGN_BF16)}};
#undef LGN_LK
#define LGN_WK(T) {reinterpret_cast<const void *>(&window_kernel<T, 1>), reinterpret_cast<const void *>(&window_kernel<T, 2>), reinterpret_cast<const void *>(&window_kernel<T, 8>)}
static const void *const kWindowTable[2][3] = {LGN_WK(LGN_F32), LGN_WK(LGN_BF16)};
#undef LGN_WK
#define LGN_RK(T, O) {reinterpret_cast<const void *>(&rows_kernel<T, O, 1>), reinterpret_cast<const void *>(&rows_kernel<T, O, 2>), reinterpret_cast<const void *>(&rows_kernel<T, O, 8>)}
static const void *const kRowTable[2][2][3] = {{LGN_RK(LGN_F32, LGN_F32), LGN_RK(LGN_F32, LGN_BF16)}, {LGN_RK(LGN_BF16, LGN_F32), LGN_RK(LGN_BF16, LGN_BF16)}};
#undef LGN_RK
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
    uint32_t span = 0;
    while (span < 8 && (1ull << span) < chunks) ++span;
    const uint64_t per = 4ull * (256u >> span), blocks = (tokens + per - 1) / per;
    if (blocks > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    uint32_t d = (uint32_t)dim, wide = ids_bits == 64;
    float s = (float)scale;
    unsigned long long *outside = reinterpret_cast<unsigned long long *>(n_outside_dev);
    log_line("embedding: %llu tokens, dim %u, %d elements per access, %llu CTAs", (unsigned long long)tokens, d, kVe[vi], (unsigned long long)blocks);
    void *args[] = {&table, &ld_table, &vocab, &d, &ids, &wide, &tokens, &s, &out, &ld_out, &span, &outside};
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
    for (int i = 0; i < 2; ++i) { s.key[i] = reinterpret_cast<uint32_t *>(w + l.key[i]); s.pos[i] = reinterpret_cast<uint32_t *>(w + l.pos[i]); }
    s.run = reinterpret_cast<uint2 *>(w + l.run);
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
    const void *sort = reinterpret_cast<const void *>(&sort_ids_kernel);
    if (cudaFuncSetAttribute(sort, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * kSortBins * 4) != cudaSuccess) { (void)cudaGetLastError(); return LGN_ERR_CUDA; }
    {
        void *args[] = {&s};
        const lgn_status r = launch_dependent(sort, dim3(kSortCtas), dim3(kSortThreads), args, smem, stream, kSortCtas);
        if (r != LGN_OK) return r;
    }
    const int vi = vector_of(dim, dout, ld_dout, ed, dtable, ld_table, et);
    SumArgs a = {};
    a.dout = dout; a.ld_dout = ld_dout;
    a.key = s.key[(s.passes + 1) & 1];
    a.pos = s.pos[(s.passes + 1) & 1];
    a.run = s.run;
    a.part = reinterpret_cast<float *>(w + l.part);
    a.out = dtable; a.ld_out = ld_table; a.vocab = vocab;
    a.tokens = s.tokens;
    a.window_log2 = l.window_log2; a.windows = l.windows;
    a.dim = (uint32_t)dim; a.pitch = l.pitch;
    a.slabs = (uint32_t)((dim + 32 * kVe[vi] - 1) / (32 * kVe[vi]));
    a.accumulate = accumulate != 0;
    a.scale = (float)scale;
    void *args[] = {&a};
    const uint64_t wblocks = ((uint64_t)l.windows * a.slabs + 7) / 8, groups = (vocab + kRowsPerWarp - 1) / kRowsPerWarp, rblocks = (groups * a.slabs + 7) / 8;
    if (wblocks > 0x7fffffffull || rblocks > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    log_line("embedding_grad: %u tokens, %llu rows, dim %u, %u passes of %u bits, %u windows, %d elements per access", s.tokens,
             (unsigned long long)vocab, a.dim, s.passes, s.bits, l.windows, kVe[vi]);
    if (l.windows > 1) {
        const lgn_status r = launch_dependent(kWindowTable[dout_dt][vi], dim3((unsigned)wblocks), dim3(256), args, 0, stream);
        if (r != LGN_OK) return r;
    }
    return launch_dependent(kRowTable[dout_dt][table_dt][vi], dim3((unsigned)rblocks), dim3(256), args, 0, stream);
}
