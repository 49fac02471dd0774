// Global gradient norm over many tensors, and clipping.
//
//   S = sum over all tensors of x^2,  norm = sqrt(S),  coef = min(1, max_norm / norm),  out = round(x coef).
//
// Bound by memory: every gradient is read for the sum and read again (from L2 for what still lies there) to
// be scaled.  Two launches for up to kClipPerLaunch tensors; the descriptors travel in the kernels' parameters.  A CTA
// takes one unit of consecutive tiles, numbered over all tensors.  norm_kernel leaves one partial sum per unit in the
// workspace.  Up to kClipSmallUnits units, every CTA of clip_kernel adds all partial sums in the same order and forms the
// coefficient itself, so that nothing has to be set up or waited for.  Above that the CTA that finishes last adds them once
// (a ticket, cleared by a memset before), and CTAs are handed out by the hardware as others end: with equal shares fixed
// beforehand the SMs differed by 20 % in speed and a pass over 1 GB took 242 us.
//
// Squares are formed and added in fp32 over one 32-byte chunk (8 or 16 values) and carried in fp64 from there
// on.  A chunk whose fp32 sum is not within [2^-80, inf), where squares may have overflowed or lost their
// low end, is added again in fp64, value by value; there the non-finite values are counted too.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_launch.h"
#include "lgn_log.h"

namespace lgn {

constexpr int kClipThreads = 256;
constexpr int kClipTileBytes = 32768;              // 4 chunks of 32 bytes per thread
constexpr int kClipPerLaunch = 512;                // tensors described in one launch's parameters
constexpr int kClipSmallList = 64;                 // ... in the parameters of the small form
constexpr uint32_t kClipSmallUnits = 592;          // units whose partial sums every CTA adds up for itself
constexpr uint32_t kClipSlots = 8192;              // units, and partial sums, per launch

struct ClipPartial { double sum; unsigned long long bad; };
struct ClipTotal { double sum; unsigned long long bad; unsigned int ticket; unsigned int pad; };

template <int N> struct ClipList {
    const char *g[N];
    char *out[N];
    uint64_t n[N];                                 // elements; bit 63: bf16
    uint32_t first[N];                             // first tile
    uint32_t count, tiles, unit;                   // unit: tiles per CTA
};

// A tensor's tiles are cut at multiples of the tile size from the 32-byte boundary at or below its first
// element, so that every chunk but the first and last is whole and aligned.
struct ClipTensor {
    const char *g;
    char *out;
    uint64_t n;
    uint32_t es, lead;                             // element size; bytes between the boundary and the first element
};

template <int N>
__device__ __forceinline__ ClipTensor clip_tensor(const ClipList<N> &l, uint32_t i) {
    ClipTensor t;
    t.g = l.g[i];
    t.out = l.out[i];
    t.es = l.n[i] >> 63 ? 2u : 4u;
    t.n = l.n[i] & ~(1ull << 63);
    t.lead = (uint32_t)(reinterpret_cast<uintptr_t>(t.g) & 31u);
    return t;
}

template <int N>
__device__ __forceinline__ uint32_t clip_find(const ClipList<N> &l, uint32_t tile) {     // the tensor a tile lies in
    uint32_t lo = 0, hi = l.count;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (l.first[mid] <= tile) lo = mid; else hi = mid;
    }
    return lo;
}

struct Words { uint32_t w[8]; };

__device__ __forceinline__ Words load_words(const char *p) {
    Words c;
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(c.w[0]), "=r"(c.w[1]), "=r"(c.w[2]), "=r"(c.w[3]), "=r"(c.w[4]), "=r"(c.w[5]), "=r"(c.w[6]), "=r"(c.w[7]) : "l"(p) : "memory");
    return c;
}
__device__ __forceinline__ Words load_words_once(const char *p) {      // memory that this kernel does not write
    Words c;
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(c.w[0]), "=r"(c.w[1]), "=r"(c.w[2]), "=r"(c.w[3]), "=r"(c.w[4]), "=r"(c.w[5]), "=r"(c.w[6]), "=r"(c.w[7]) : "l"(p) : "memory");
    return c;
}
__device__ __forceinline__ void prefetch_l2(const char *p) { asm volatile("prefetch.global.L2 [%0];" :: "l"(p)); }
__device__ __forceinline__ void store_words(char *p, const Words &c) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(c.w[0]), "r"(c.w[1]), "r"(c.w[2]), "r"(c.w[3]), "r"(c.w[4]), "r"(c.w[5]), "r"(c.w[6]), "r"(c.w[7]) : "memory");
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// One word (one or two values) in fp64.  Everything by value: a chunk passed by reference to a function that is not inlined
// would live in local memory on the fast path too.
template <int ES>
__device__ __noinline__ double square_exactly(uint32_t w) {
    const float a = ES == 4 ? __uint_as_float(w) : bf_lo(w), b = ES == 4 ? 0.0f : bf_hi(w);
    return (double)a * (double)a + (double)b * (double)b;
}
template <int ES>
__device__ __forceinline__ unsigned int non_finite(uint32_t w) {
    if constexpr (ES == 4) return (w & 0x7f800000u) == 0x7f800000u;
    else return ((w & 0x7f80u) == 0x7f80u) + ((w & 0x7f800000u) == 0x7f800000u);
}

template <int ES>
__device__ __forceinline__ void add_exactly(const Words &c, double &sum, unsigned long long &bad) {
    unsigned int n = 0;
    #pragma unroll
    for (int k = 0; k < 8; ++k) { sum += square_exactly<ES>(c.w[k]); n += non_finite<ES>(c.w[k]); }
    bad += n;
}

template <int ES>
__device__ __forceinline__ void add_chunk(const Words &c, double &sum, unsigned long long &bad) {
    float s = 0.0f, t = 0.0f;
    #pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (ES == 4) {
            if (k & 1) t = fmaf(__uint_as_float(c.w[k]), __uint_as_float(c.w[k]), t);
            else       s = fmaf(__uint_as_float(c.w[k]), __uint_as_float(c.w[k]), s);
        } else {
            s = fmaf(bf_lo(c.w[k]), bf_lo(c.w[k]), s);
            t = fmaf(bf_hi(c.w[k]), bf_hi(c.w[k]), t);
        }
    }
    s += t;
    if (s >= 0x1p-80f && s < __int_as_float(0x7f800000)) sum += (double)s;
    else {
        uint32_t bits = 0;                                 // all zeros, as in pruned gradients: nothing to add (85 % zeros in bf16: 140 -> 85 us per 537 MB)
        #pragma unroll
        for (int k = 0; k < 8; ++k) bits |= c.w[k] & (ES == 4 ? 0x7fffffffu : 0x7fff7fffu);
        if (bits != 0) add_exactly<ES>(c, sum, bad);
    }
}

__device__ __forceinline__ float load_elem(const char *p, uint32_t es) {
    return es == 4 ? *reinterpret_cast<const float *>(p) : __uint_as_float((uint32_t)*reinterpret_cast<const unsigned short *>(p) << 16);
}

// Word k of chunk number c of a tensor with the values outside it as zeros.
__device__ __noinline__ uint32_t load_edge_word(const char *g, uint64_t n, uint32_t es, uint32_t lead, uint64_t c, int k) {
    const int64_t at = (int64_t)(c * 32) - lead + 4 * k, end = (int64_t)(n * es);        // byte offset from the first element
    if (es == 4) return at >= 0 && at < end ? *reinterpret_cast<const uint32_t *>(g + at) : 0u;
    uint32_t w = at >= 0 && at < end ? *reinterpret_cast<const unsigned short *>(g + at) : 0u;
    if (at + 2 >= 0 && at + 2 < end) w |= (uint32_t)*reinterpret_cast<const unsigned short *>(g + at + 2) << 16;
    return w;
}
__device__ __forceinline__ Words load_edge(const ClipTensor &t, uint64_t c) {
    Words w;
    #pragma unroll
    for (int k = 0; k < 8; ++k) w.w[k] = load_edge_word(t.g, t.n, t.es, t.lead, c, k);
    return w;
}

__device__ __forceinline__ double block_sum(double v, unsigned long long &bad, double *sh, unsigned long long *shb) {
    #pragma unroll
    for (int d = 16; d; d >>= 1) {
        v += __shfl_down_sync(0xffffffffu, v, d);
        bad += __shfl_down_sync(0xffffffffu, bad, d);
    }
    if ((threadIdx.x & 31) == 0) { sh[threadIdx.x >> 5] = v; shb[threadIdx.x >> 5] = bad; }
    __syncthreads();
    double s = 0.0;
    unsigned long long b = 0;
    #pragma unroll
    for (int w = 0; w < kClipThreads / 32; ++w) { s += sh[w]; b += shb[w]; }
    bad = b;
    return s;
}

// Tiles [t, stop) of one tensor, whose first tile is `first`.  The tile after the current one is asked for in L2.
template <int ES>
__device__ __forceinline__ void add_tiles(const ClipTensor &x, uint32_t first, uint32_t t, uint32_t stop, double &sum, unsigned long long &bad) {
    const uint64_t bytes = x.lead + x.n * ES, whole = bytes / 32;                    // chunks [1 if lead, whole) lie inside
    const char *base = x.g - x.lead;
    for (; t < stop; ++t) {
        const uint64_t c0 = (uint64_t)(t - first) * (kClipTileBytes / 32) + threadIdx.x;
        if ((t != first || x.lead == 0) && (uint64_t)(t - first + 1) * (kClipTileBytes / 32) <= whole) {
            Words c[4];
            #pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = load_words_once(base + (c0 + k * kClipThreads) * 32);
            if (t + 1 < stop && (uint64_t)(t - first + 2) * (kClipTileBytes / 32) <= whole) {
                #pragma unroll
                for (int k = 0; k < 4; ++k) prefetch_l2(base + (c0 + (k + 4) * kClipThreads) * 32);
            }
            #pragma unroll
            for (int k = 0; k < 4; ++k) add_chunk<ES>(c[k], sum, bad);
        } else {
            for (int k = 0; k < 4; ++k) {
                const uint64_t at = c0 + k * kClipThreads;
                if (at < whole && !(at == 0 && x.lead != 0)) add_chunk<ES>(load_words(base + at * 32), sum, bad);
                else if (at * 32 < bytes) add_exactly<ES>(load_edge(x, at), sum, bad);
            }
        }
    }
}

// total == nullptr: only the partial sums.  slot0: the first partial sum of this launch; all: those of every launch so far.
template <int N>
__global__ void __launch_bounds__(kClipThreads, 4)
norm_kernel(const __grid_constant__ ClipList<N> l, ClipPartial *part, uint32_t slot0, ClipTotal *total) {
    __shared__ double sh[kClipThreads / 32];
    __shared__ unsigned long long shb[kClipThreads / 32];
    __shared__ uint32_t last;
    dep_launch();
    dep_wait();
    const uint32_t t0 = blockIdx.x * l.unit, t1 = min(l.tiles, t0 + l.unit);
    double sum = 0.0;
    unsigned long long bad = 0;
    if (t0 < t1) {
        uint32_t i = clip_find(l, t0);
        for (uint32_t t = t0; t < t1; ++i) {
            const ClipTensor x = clip_tensor(l, i);
            const uint32_t stop = min(t1, i + 1 < l.count ? l.first[i + 1] : l.tiles);
            if (x.es == 4) add_tiles<4>(x, l.first[i], t, stop, sum, bad);
            else           add_tiles<2>(x, l.first[i], t, stop, sum, bad);
            t = stop;
        }
    }
    sum = block_sum(sum, bad, sh, shb);
    if (threadIdx.x == 0) { part[slot0 + blockIdx.x].sum = sum; part[slot0 + blockIdx.x].bad = bad; }
    if (total == nullptr) return;
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&total->ticket, 1u) + 1u == gridDim.x;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    bad = 0;
    for (uint32_t i = threadIdx.x; i < slot0 + gridDim.x; i += kClipThreads) { sum += __ldcg(&part[i].sum); bad += __ldcg(&part[i].bad); }
    __syncthreads();
    sum = block_sum(sum, bad, sh, shb);
    if (threadIdx.x == 0) { total->sum = sum; total->bad = bad; }
}

__device__ __forceinline__ float clip_coef(double sum, double max_norm, bool clip) {
    const double norm = sqrt(sum);
    return clip && norm > max_norm && norm < __longlong_as_double(0x7ff0000000000000ll) ? (float)(max_norm / norm) : 1.0f;
}

template <int ES>
__device__ __forceinline__ Words scaled_words(const Words &c, float coef) {
    Words r;
    #pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (ES == 4) r.w[k] = __float_as_uint(__uint_as_float(c.w[k]) * coef);
        else {
            const __nv_bfloat162 p = __floats2bfloat162_rn(bf_lo(c.w[k]) * coef, bf_hi(c.w[k]) * coef);
            r.w[k] = *reinterpret_cast<const uint32_t *>(&p);
        }
    }
    return r;
}

// Elements at byte offsets [lo, hi) from the first one, value by value.
template <int ES>
__device__ __noinline__ void scale_elements(const ClipTensor x, int64_t lo, int64_t hi, uint32_t first, uint32_t step, float coef) {
    const int64_t end = (int64_t)(x.n * ES), from = lo < 0 ? 0 : lo, to = hi < end ? hi : end;
    for (int64_t p = from + (int64_t)first * ES; p < to; p += (int64_t)step * ES) {
        const float v = load_elem(x.g + p, ES) * coef;
        if constexpr (ES == 4) *reinterpret_cast<float *>(x.out + p) = v;
        else *reinterpret_cast<__nv_bfloat16 *>(x.out + p) = __float2bfloat16_rn(v);
    }
}

// Tiles [stop, t) of one tensor, whose first tile is `first`, from the last to the first.
template <int ES>
__device__ __forceinline__ void scale_tiles(const ClipTensor &x, uint32_t first, uint32_t t, uint32_t stop, float coef) {
    const uint64_t bytes = x.lead + x.n * ES, whole = bytes / 32;
    const char *base = x.g - x.lead;
    char *obase = x.out - x.lead;
    const bool same = ((reinterpret_cast<uintptr_t>(x.out) ^ reinterpret_cast<uintptr_t>(x.g)) & 31u) == 0;
    for (; t > stop; --t) {
        const uint64_t c0 = (uint64_t)(t - 1 - first) * (kClipTileBytes / 32) + threadIdx.x;
        if (!same) {                                          // input and output aligned differently: value by value, coalesced
            const int64_t lo = (int64_t)(t - 1 - first) * kClipTileBytes - x.lead;
            scale_elements<ES>(x, lo, lo + kClipTileBytes, threadIdx.x, kClipThreads, coef);
        } else if ((t - 1 != first || x.lead == 0) && (uint64_t)(t - first) * (kClipTileBytes / 32) <= whole) {
            Words c[4];
            #pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = load_words(base + (c0 + k * kClipThreads) * 32);
            if (t - 1 > stop && t - 2 != first) {
                #pragma unroll
                for (int k = 0; k < 4; ++k) prefetch_l2(base + (c0 + (k - 4) * kClipThreads) * 32);
            }
            #pragma unroll
            for (int k = 0; k < 4; ++k) store_words(obase + (c0 + k * kClipThreads) * 32, scaled_words<ES>(c[k], coef));
        } else {
            for (int k = 0; k < 4; ++k) {
                const uint64_t at = c0 + k * kClipThreads;
                if (at < whole && !(at == 0 && x.lead != 0)) store_words(obase + at * 32, scaled_words<ES>(load_words(base + at * 32), coef));
                else if (at * 32 < bytes) scale_elements<ES>(x, (int64_t)(at * 32) - x.lead, (int64_t)(at * 32 + 32) - x.lead, 0, 1, coef);
            }
        }
    }
}

// SCALE: scale (or, for a coefficient of 1, copy) every tensor; otherwise only the record is written.  The sum of
// squares is the record's (from_record: a caller may have reduced it over ranks), or `total`, or that of the partial sums.
template <int N, bool SCALE>
__global__ void __launch_bounds__(kClipThreads, 4)
clip_kernel(const __grid_constant__ ClipList<N> l, const ClipPartial *part, uint32_t nparts, const ClipTotal *total, double max_norm,
            uint32_t clip, uint32_t from_record, uint32_t write_record, lgn_norm_t *record) {
    __shared__ double sh[kClipThreads / 32];
    __shared__ unsigned long long shb[kClipThreads / 32];
    dep_launch();
    dep_wait();
    double sum = 0.0;
    unsigned long long bad = 0;
    if (from_record) {
        sum = record->sum_sq;
        bad = record->n_nonfinite;
    } else if (total != nullptr) {
        sum = total->sum;
        bad = total->bad;
    } else {
        for (uint32_t i = threadIdx.x; i < nparts; i += kClipThreads) { sum += part[i].sum; bad += part[i].bad; }
        sum = block_sum(sum, bad, sh, shb);
    }
    const float coef = clip_coef(sum, max_norm, clip != 0);
    if (blockIdx.x == 0 && threadIdx.x == 0 && write_record) {
        record->norm = (float)sqrt(sum);
        record->coef = coef;
        if (!from_record) { record->n_nonfinite = bad; record->sum_sq = sum; }
    }
    if constexpr (SCALE) {
        // from the last tile to the first: the order in which L2 still holds them
        const uint32_t t0 = (gridDim.x - 1 - blockIdx.x) * l.unit, t1 = min(l.tiles, t0 + l.unit);
        if (t0 >= t1) return;
        uint32_t i = clip_find(l, t1 - 1);
        for (uint32_t t = t1; t > t0; --i) {
            const ClipTensor x = clip_tensor(l, i);
            const uint32_t stop = max(t0, l.first[i]);
            if (coef != 1.0f || x.out != x.g) {
                if (x.es == 4) scale_tiles<4>(x, l.first[i], t, stop, coef);
                else           scale_tiles<2>(x, l.first[i], t, stop, coef);
            }
            t = stop;
        }
    }
}

template <int N>
static void fill_list(ClipList<N> &l, const lgn_grad_t *grads, int count) {
    uint32_t tiles = 0, c = 0;
    for (int i = 0; i < count; ++i) {
        if (grads[i].n == 0) continue;
        const uint64_t es = grads[i].dt == LGN_BF16 ? 2 : 4;
        l.g[c] = static_cast<const char *>(grads[i].g);
        l.out[c] = static_cast<char *>(grads[i].out);
        l.n[c] = grads[i].n | (grads[i].dt == LGN_BF16 ? 1ull << 63 : 0ull);
        l.first[c] = tiles;
        tiles += (uint32_t)(((reinterpret_cast<uintptr_t>(grads[i].g) & 31u) + grads[i].n * es + kClipTileBytes - 1) / kClipTileBytes);
        ++c;
    }
    l.count = c;
    l.tiles = tiles;
}

// Tiles per CTA: one while that gives at most kClipSmallUnits units, else eight (256 KiB) or as many as keep
// the units within their slots.
static uint32_t unit_of(uint64_t tiles) {
    if (tiles <= kClipSmallUnits) return 1;
    const uint64_t need = (tiles + kClipSlots - 1) / kClipSlots;
    return (uint32_t)(need < 8 ? 8 : need);
}

struct ClipCall {
    double max_norm;
    uint32_t clip, from_record;
    bool norm, scale, ticket;
    lgn_norm_t *record;
    ClipPartial *part;
    ClipTotal *total;
    void *stream;
};

template <int N>
static lgn_status run_pass(const lgn_grad_t *grads, int count, const ClipCall &k, bool second, bool last, uint32_t slot, uint32_t &slots, bool write_record, uint32_t nparts) {
    ClipList<N> l;
    fill_list(l, grads, count);
    l.unit = unit_of(l.tiles);
    uint32_t grid = (l.tiles + l.unit - 1) / l.unit;
    if (grid < 1) grid = 1;
    ClipPartial *part = k.part;
    if (!second) {
        ClipTotal *total = k.ticket && last ? k.total : nullptr;
        void *args[] = {&l, &part, &slot, &total};
        slots = grid;
        return launch_dependent(reinterpret_cast<const void *>(&norm_kernel<N>), dim3(grid), dim3(kClipThreads), args, 0, k.stream);
    }
    const ClipTotal *total = k.ticket ? k.total : nullptr;
    double max_norm = k.max_norm;
    uint32_t clip = k.clip, from = k.from_record, write = write_record;
    lgn_norm_t *record = k.record;
    void *args[] = {&l, &part, &nparts, &total, &max_norm, &clip, &from, &write, &record};
    if (k.scale) return launch_dependent(reinterpret_cast<const void *>(&clip_kernel<N, true>), dim3(grid), dim3(kClipThreads), args, 0, k.stream);
    return launch_dependent(reinterpret_cast<const void *>(&clip_kernel<N, false>), dim3(1), dim3(kClipThreads), args, 0, k.stream);
}

static uint64_t tiles_of(const lgn_grad_t &x) {
    const uint64_t es = x.dt == LGN_BF16 ? 2 : 4;
    return x.n == 0 ? 0 : ((reinterpret_cast<uintptr_t>(x.g) & 31u) + x.n * es + kClipTileBytes - 1) / kClipTileBytes;
}

static lgn_status run_clip(const lgn_grad_t *grads, int count, ClipCall k) {
    uint64_t tiles = 0;
    for (int i = 0; i < count; ++i) tiles += tiles_of(grads[i]);
    k.ticket = k.norm && (tiles > kClipSmallUnits || count > kClipPerLaunch);
    log_line("clip: %d tensors, %llu tiles, %s", count, (unsigned long long)tiles, k.ticket ? "sum by the last CTA" : "sum by every CTA");
    if (k.ticket && cudaMemsetAsync(k.total, 0, sizeof *k.total, static_cast<cudaStream_t>(k.stream)) != cudaSuccess) {
        (void)cudaGetLastError();
        return LGN_ERR_CUDA;
    }
    uint32_t slot = 0, slots = 0;
    for (int pass = k.norm ? 0 : 1; pass < 2; ++pass) {
        for (int i = 0; i == 0 || i < count; i += kClipPerLaunch) {
            const int c = count - i < kClipPerLaunch ? count - i : kClipPerLaunch;
            const bool last = i + kClipPerLaunch >= count;
            const lgn_status s = c <= kClipSmallList ? run_pass<kClipSmallList>(grads + i, c, k, pass == 1, last, slot, slots, i == 0, slot)
                                                     : run_pass<kClipPerLaunch>(grads + i, c, k, pass == 1, last, slot, slots, i == 0, slot);
            if (s != LGN_OK) return s;
            if (pass == 0) slot += slots;
            else if (!k.scale) break;
        }
    }
    return LGN_OK;
}

static lgn_status check_grads(const lgn_grad_t *grads, int count, bool with_out) {
    if (count < 0 || (count > 0 && grads == nullptr)) return LGN_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        const lgn_grad_t &x = grads[i];
        if ((x.dt != LGN_F32 && x.dt != LGN_BF16) || x.reserved != 0) return LGN_ERR_INVALID_ARG;
        if (x.n > (1ull << 40)) return LGN_ERR_UNSUPPORTED;
        if (x.n == 0) continue;
        const uint64_t es = x.dt == LGN_BF16 ? 2 : 4;
        if (x.g == nullptr || !aligned_to(x.g, es)) return LGN_ERR_INVALID_ARG;
        if (!with_out) continue;
        if (x.out == nullptr || !aligned_to(x.out, es)) return LGN_ERR_INVALID_ARG;
        if (x.out != x.g && ranges_overlap(x.g, x.n * es, x.out, x.n * es)) return LGN_ERR_INVALID_ARG;
    }
    // the tile numbers of one launch are 32 bits wide
    for (int i = 0; i < count; i += kClipPerLaunch) {
        uint64_t tiles = 0;
        for (int j = i; j < count && j < i + kClipPerLaunch; ++j) tiles += (grads[j].n * (grads[j].dt == LGN_BF16 ? 2 : 4)) / kClipTileBytes + 2;
        if (tiles > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    }
    return LGN_OK;
}

}  // namespace lgn

using namespace lgn;

extern "C" size_t lgn_clip_workspace_bytes(int count) {
    if (count < 0) return 0;
    const size_t launches = count == 0 ? 1 : ((size_t)count + kClipPerLaunch - 1) / kClipPerLaunch;
    return launches * kClipSlots * sizeof(ClipPartial) + sizeof(ClipTotal);
}

static lgn_status norm_and_clip(const lgn_grad_t *grads, int count, double max_norm, bool clip, lgn_norm_t *record, void *ws, size_t ws_bytes, void *stream) {
    const lgn_status s = check_grads(grads, count, clip);
    if (s != LGN_OK) return s;
    if (clip && !(max_norm >= 0.0)) return LGN_ERR_INVALID_ARG;
    if (record == nullptr || !aligned_to(record, 8) || ws == nullptr || !aligned_to(ws, 16)) return LGN_ERR_INVALID_ARG;
    if (ws_bytes < lgn_clip_workspace_bytes(count)) return LGN_ERR_WORKSPACE;
    ClipTotal *total = static_cast<ClipTotal *>(ws);
    const ClipCall k = {max_norm, clip, 0, true, clip, false, record, reinterpret_cast<ClipPartial *>(total + 1), total, stream};
    return run_clip(grads, count, k);
}

extern "C" lgn_status lgn_grad_norm(const lgn_grad_t *grads, int count, lgn_norm_t *record_dev, void *ws, size_t ws_bytes, void *stream) {
    return norm_and_clip(grads, count, 0.0, false, record_dev, ws, ws_bytes, stream);
}

extern "C" lgn_status lgn_clip_grad_norm(const lgn_grad_t *grads, int count, double max_norm, lgn_norm_t *record_dev, void *ws, size_t ws_bytes, void *stream) {
    return norm_and_clip(grads, count, max_norm, true, record_dev, ws, ws_bytes, stream);
}

extern "C" lgn_status lgn_clip_apply(const lgn_grad_t *grads, int count, double max_norm, lgn_norm_t *record_dev, void *stream) {
    const lgn_status s = check_grads(grads, count, true);
    if (s != LGN_OK) return s;
    if (!(max_norm >= 0.0) || record_dev == nullptr || !aligned_to(record_dev, 8)) return LGN_ERR_INVALID_ARG;
    const ClipCall k = {max_norm, 1, 1, false, true, false, record_dev, nullptr, nullptr, stream};
    return run_clip(grads, count, k);
}
