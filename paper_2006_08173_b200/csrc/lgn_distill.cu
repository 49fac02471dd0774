// Loss of a student's logits s against a teacher's top logits z at places id, and its gradient, row by row:
//
//   p = softmax(z / T) over the places present,   q = softmax(s / T),   q1 = softmax(s)
//   loss = a T^2 sum p (ln p - ln q[id]) + (1 - a) (-ln q1[label])
//   ds   = w (a T (q - p at id) + (1 - a) (q1 - 1 at label))
//
// With M = max s, S = sum exp((s - M) / T) and Z, zm the same of the teacher, the first part is
//   a T (1/Z sum exp((z - zm) / T) ((z - zm) - (s[id] - M))) + a T^2 (ln S - ln Z),
// so a row needs one pass for M and the sums and, for the gradient, one more.  A gradient keeps its row in shared memory in between:
// 32, 64 or 128 threads with up to 16 pieces of 16 bytes each, or a cluster of up to 8 such CTAs (their sums are joined through
// distributed shared memory); rows beyond that go through in chunks that are read again, from L2 mostly.  The loss alone takes
// chunks of 8 pieces per thread straight to registers.
//
// What bounds it (calls back to back; one after other work takes 2 to 5 % longer, and two GPUs differ by as much): for one temperature the instructions
// (15 per value, 437 to 446 us for 4096 x 131072 bf16, 0.73 of the copy rate), fp32 logits the memory (8192 x 32000: 365 to 386 us, 0.83 to 0.88).  Two
// temperatures take four exponentials per value, 472 us of the special-function units alone: one of
// the gradient's two is a polynomial for three values in four of bf16 logits (4096 x 131072: 550 to 558 us, 573 to 600 after other work; on one GPU 550, all of them 562, half 562;
// with half of the first pass's too, the instructions bind: 599).  Which values those are goes by the place within 16 aligned bytes, so a value's last bits
// before the rounding to bf16 go by its column and by the row's alignment; 2.9e-6 is below a thousandth of that rounding.
// Rows beyond a cluster are read twice: 4096 x 140000 fp32 1060 us, 0.66.
// Arithmetic is on two values at a time.  Not kept: reading the row a second time from L2 instead of holding it (638 us,
// 506 for one temperature), and CTAs that stay for several rows and ask for the next as slots of the last fall free (722 and 477: more instructions
// and registers, 104 clusters at once).
//
// exp is taken in base 2 of (s - M) log2(e) / T, the difference first: it is exact or small where the term
// counts.  Sums are fp32, a few dozen terms per thread, then by lanes, warps and ranks in a fixed order.
//
// The gradient's places are written last, over what the pass wrote there.  A place that several entries name is found by a table of the ids
// in shared memory, and then summed in the order of the entries by each of them, so that all write the same value; the label
// writes its place where no entry does.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_launch.h"
#include "lgn_log.h"
#include "lgn_tensor.cuh"
#include "lgn_values.cuh"

namespace lgn {

constexpr uint64_t kDsMaxTop = 1024, kDsMaxDim = 1ull << 30;
constexpr int kDsVecs = 16;                             // pieces of 16 bytes a thread holds at most
constexpr int kDsMaxSmem = 64 * 1024;                   // above the most that a CTA asks for: 3 x 1025 + 4096 words of entries, 128 x 16 pieces
constexpr int kDsStatic = 1024;                         // above what the kernels declare: 7 sums of up to 8 warps and 3 of the CTA, 236 bytes
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kDsLowest = -3.402823466e38f;           // starts every maximum: s - M is then never inf - inf for s = -inf

struct DistillArgs {
    const char *logits;
    char *dlogits;
    const void *ids, *labels;
    const char *teacher;
    const float *weight;
    float *loss;
    uint64_t ld, ldd, ld_ids, ld_teacher;
    uint32_t vocab, top;
    uint32_t pieces;                                    // of 16 bytes, per CTA of a row
    uint32_t table;                                     // slots of the id table, a power of two
    uint32_t vecs;                                      // pieces of a thread in a chunk
    uint32_t slots;                                     // where the row's pieces begin in shared memory, in words
    int32_t ids64, labels64, teacher_dt;
    float temperature, alpha, beta;                     // beta = 1 - alpha
    float scale, scale1;                                // log2(e) / T and log2(e); the first alone where one softmax serves
};

__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Two fp32 values in a register pair, and arithmetic on both at once: half the instructions.
struct Two { uint64_t w; };
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.w) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void apart(Two x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.w)); }
__device__ __forceinline__ Two operator+(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
    return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
    return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.w) : "l"(a.w), "l"(b.w), "l"(c.w));
    return r;
}
__device__ __forceinline__ Two exp2_approx(Two x) {
    float a, b;
    apart(x, a, b);
    return two(exp2_approx(a), exp2_approx(b));
}
// 2^x for x <= 0 on the multiply-add pipes: x is split into a whole number n (added to 1.5 2^23 it stands in the low bits) and f in [-1/2, 1/2], 2^f is
// a polynomial (constant term 1, the rest fitted for the least relative error, 2.9e-6 with its roundings), and n is added to its exponent.
// From -127 on down: zero.  Not for NaN.
__device__ __forceinline__ Two exp2_poly(Two x) {
    float a, b, c, d;
    apart(x, a, b);
    x = two(fmaxf(a, -127.0f), fmaxf(b, -127.0f));
    const Two r = x + two(12582912.0f, 12582912.0f), f = fma(r + two(-12582912.0f, -12582912.0f), two(-1.0f, -1.0f), x);
    Two y = fma(f, two(0.009582853f, 0.009582853f), two(0.055906426f, 0.055906426f));
    y = fma(f, y, two(0.24024099f, 0.24024099f));
    y = fma(f, y, two(0.6931242f, 0.6931242f));
    y = fma(f, y, two(1.0f, 1.0f));
    apart(r, a, b);
    apart(y, c, d);
    return two(__uint_as_float((__float_as_uint(a) << 23) + __float_as_uint(c)), __uint_as_float((__float_as_uint(b) << 23) + __float_as_uint(d)));
}
template <int DT>
__device__ __forceinline__ float ds_load(const char *p, uint64_t i) {
    if constexpr (DT == LGN_F32) return __uint_as_float(ldro_u32(p + 4 * i));
    else return __uint_as_float(ldro_u16(p + 2 * i) << 16);
}
__device__ __forceinline__ int64_t ds_id(const void *ids, int is64, uint64_t i) {
    return is64 ? (int64_t)ldro_u64(static_cast<const char *>(ids) + 8 * i) : (int64_t)(int32_t)ldro_u32(static_cast<const char *>(ids) + 4 * i);
}
template <int DT>
__device__ __forceinline__ void ds_store(char *p, uint64_t i, float v) {
    if constexpr (DT == LGN_F32) reinterpret_cast<float *>(p)[i] = v;
    else reinterpret_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// 16 bytes of a row as they lie in memory.
template <int DT> struct Piece {
    static constexpr int kVals = DT == LGN_F32 ? 4 : 8;
    uint32_t w[4];
    __device__ __forceinline__ float at(int k) const {
        if constexpr (DT == LGN_F32) return __uint_as_float(w[k]);
        else return k & 1 ? bf_hi(w[k >> 1]) : bf_lo(w[k >> 1]);
    }
    __device__ __forceinline__ Two pair(int k) const { return two(at(2 * k), at(2 * k + 1)); }
    __device__ __forceinline__ float max_with(float m) const {           // bf16 in pairs
        if constexpr (DT == LGN_F32) return fmaxf(fmaxf(m, fmaxf(at(0), at(1))), fmaxf(at(2), at(3)));
        else {
            uint32_t a, b;
            asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(w[0]), "r"(w[1]));
            asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(w[2]), "r"(w[3]));
            asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
            return fmaxf(m, fmaxf(bf_lo(a), bf_hi(a)));
        }
    }
    // What was made of the words so far is not kept for later: unpacked values would take twice the registers.
    __device__ __forceinline__ void forget() { asm volatile("" : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])); }
};
// A piece that the row begins or ends in: column `c` is the first, columns outside the row read as -inf and are not written.  Of its own, so that
// the loops over whole pieces stay short.
template <int DT>
__device__ __noinline__ uint4 load_edge(const char *row, int64_t c, uint32_t vocab) {
    uint32_t w[4];
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DT == LGN_F32) {
            w[k] = c + k >= 0 && c + k < (int64_t)vocab ? ldro_u32(row + (c + k) * 4) : 0xff800000u;
        } else {
            w[k] = c + 2 * k >= 0 && c + 2 * k < (int64_t)vocab ? ldro_u16(row + (c + 2 * k) * 2) : 0xff80u;
            w[k] |= (c + 2 * k + 1 >= 0 && c + 2 * k + 1 < (int64_t)vocab ? ldro_u16(row + (c + 2 * k + 1) * 2) : 0xff80u) << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The same for a gradient that is aligned differently from its logits.
template <int DT>
__device__ __noinline__ void store_edge(char *row, int64_t c, uint32_t vocab, uint4 q) {
    constexpr int ES = DT == LGN_F32 ? 4 : 2, kVals = 16 / ES;
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    #pragma unroll
    for (int k = 0; k < kVals; ++k) {
        if (c + k < 0 || c + k >= (int64_t)vocab) continue;
        if constexpr (DT == LGN_F32) *reinterpret_cast<uint32_t *>(row + (c + k) * ES) = w[k];
        else *reinterpret_cast<uint16_t *>(row + (c + k) * ES) = (uint16_t)(k & 1 ? w[k >> 1] >> 16 : w[k >> 1]);
    }
}

__device__ __forceinline__ float shared_of(uint32_t addr, uint32_t rank) {
    uint32_t at;
    float x;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
    return x;
}

__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
template <int WIDTH>
__device__ __forceinline__ float lanes_sum(float v) {
    #pragma unroll
    for (int d = WIDTH / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// What is known of a teacher's entries: their maximum, sum and weighted differences dot = sum exp((z - zm) / T) ((z - zm) - (s - sm)), sm the largest
// of the student's logits at the places.
struct TeacherSums {
    float zm, sm, sum, dot;
    __device__ __forceinline__ void rebase(float z, float s, float scale) {
        const float f = sum != 0.0f ? exp2_approx((zm - z) * scale) : 0.0f;         // without entries the references mean nothing
        dot = f != 0.0f ? f * (dot + sum * ((zm - z) - (sm - s))) : 0.0f;
        sum *= f;
        zm = z;
        sm = s;
    }
    __device__ __forceinline__ void add(float z, float s, float scale) {
        rebase(fmaxf(zm, z), fmaxf(sm, s), scale);
        const float e = exp2_approx((z - zm) * scale);
        sum += e;
        if (e != 0.0f) dot += e * ((z - zm) - (s - sm));
    }
    // Over groups of WIDTH lanes (copies of one another beyond the first), in a fixed order.
    template <int WIDTH>
    __device__ __forceinline__ void join(float scale) {
        rebase(warp_max(zm), warp_max(sm), scale);
        sum = lanes_sum<WIDTH>(sum);
        dot = lanes_sum<WIDTH>(dot);
    }
};

// DUAL: the two parts take softmaxes of different temperatures.
template <int DT, int THREADS, bool DUAL, bool GRAD>
__global__ void __launch_bounds__(THREADS, THREADS == 32 ? 32 : GRAD ? 768 / THREADS : 1024 / THREADS)
distill_kernel(const DistillArgs p) {
    constexpr int kVals = Piece<DT>::kVals, ES = 16 / kVals, kWarps = THREADS / 32;
    extern __shared__ uint32_t dyn[];
    __shared__ float parts[7][kWarps];
    __shared__ float joint[3];
    dep_launch();

    uint32_t rank, nrank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(nrank));
    const uint64_t row = blockIdx.x / nrank;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t entries = p.top + 1;                 // the label is the last
    int32_t *id = reinterpret_cast<int32_t *>(dyn);     // -1: absent
    float *ze = reinterpret_cast<float *>(dyn + entries), *se = ze + entries;
    uint32_t *table = dyn + 3 * entries;                // id + 1, the top bit: named more than once
    if constexpr (GRAD) {
        for (uint32_t i = tid; i < p.table; i += THREADS) table[i] = 0u;
        __syncthreads();
    }
    dep_wait();

    const char *src = p.logits + row * p.ld * ES;
    char *dst = GRAD ? p.dlogits + row * p.ldd * ES : nullptr;
    const int64_t shift = (int64_t)((reinterpret_cast<uintptr_t>(src) & 15) / ES), vocab = (int64_t)p.vocab;
    const bool alike = GRAD && ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0;
    const uint32_t total = (uint32_t)((shift + vocab + kVals - 1) / kVals);             // pieces of the row
    const uint32_t v0 = min(rank * p.pieces, total), v1 = min(v0 + p.pieces, total);
    const uint32_t in0 = shift > 0 ? 1u : 0u, in1 = max(in0, min(v1, (uint32_t)((shift + vocab) / kVals)));   // whole pieces
    const char *base = src - shift * ES;

    // An entry: its place, the teacher's logit, the student's.
    auto place_of = [&](uint32_t j, float &z) {
        int64_t at = -1;
        if (j < p.top) {
            at = ds_id(p.ids, p.ids64, row * p.ld_ids + j);
            z = p.teacher_dt == LGN_F32 ? ds_load<LGN_F32>(p.teacher, row * p.ld_teacher + j) : ds_load<LGN_BF16>(p.teacher, row * p.ld_teacher + j);
        } else if (j == p.top && p.labels != nullptr) at = ds_id(p.labels, p.labels64, row);
        return at;
    };
    auto present = [&](uint32_t j, int64_t at, float z) {
        if (at < 0 || at >= vocab) return -1;
        return (j < p.top ? z == -INFINITY || p.alpha == 0.0f : p.beta == 0.0f) ? -1 : (int32_t)at;
    };
    // Loads are issued ahead of what waits for them: the thread's first entry, the row's first chunk, the entry's logit.
    float z0 = 0.0f, s0 = 0.0f, w = 1.0f;
    const int64_t far0 = place_of(tid, z0);
    if (GRAD && p.weight != nullptr) w = __uint_as_float(ldro_u32(p.weight + row));
    const uint32_t slots = smem_u32(dyn + p.slots) + tid * 16;      // the thread's pieces: nobody else's, no barrier
    // Pieces of a thread in the chunk from v on: `all` of them, of which [skip, whole) are whole and at most one on either side is not.
    uint32_t all, skip, whole;
    auto count = [&](uint32_t v) {
        const uint32_t u = v + tid, end = min(v1, v + THREADS * p.vecs), last = min(end, in1);
        all = u < end ? (end - u + THREADS - 1) / THREADS : 0u;
        whole = u < last ? (last - u + THREADS - 1) / THREADS : 0u;
        skip = u < min(in0, end) ? 1u : 0u;
    };
    auto edge = [&](uint32_t u) { return load_edge<DT>(src, (int64_t)u * kVals - shift, p.vocab); };
    // A gradient reads the row twice and keeps it in shared memory; a loss alone takes each chunk straight to registers.
    constexpr uint32_t kHeld = GRAD ? 1 : kDsVecs / 2, kStride = THREADS * 16;
    Piece<DT> held[kHeld];
    auto load = [&](uint32_t v) {
        count(v);
        const char *at = base + (uint64_t)(v + tid) * 16;
        if constexpr (GRAD) {
            auto put = [&](uint32_t i) {
                const uint4 e = edge(v + i * THREADS + tid);
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(slots + i * kStride), "r"(e.x), "r"(e.y), "r"(e.z), "r"(e.w) : "memory");
            };
            uint32_t slot = slots + skip * kStride;
            at += skip * kStride;
            #pragma unroll 4
            for (uint32_t i = skip; i < whole; ++i, slot += kStride, at += kStride)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(slot), "l"(at) : "memory");
            if (skip != 0u) put(0);
            if (whole < all) put(whole);
        } else {
            auto get = [&](uint32_t i) {
                uint32_t (&q)[4] = held[i].w;
                asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "l"(at + i * kStride) : "memory");
            };
            if (skip == 0u && whole == kHeld) {
                #pragma unroll
                for (uint32_t i = 0; i < kHeld; ++i) get(i);
            } else {
                #pragma unroll
                for (uint32_t i = 0; i < kHeld; ++i) {
                    if (i >= all) break;
                    if (i >= skip && i < whole) get(i);
                    else {
                        const uint4 e = edge(v + i * THREADS + tid);
                        held[i].w[0] = e.x; held[i].w[1] = e.y; held[i].w[2] = e.z; held[i].w[3] = e.w;
                    }
                }
            }
        }
    };
    auto piece = [&](uint32_t slot) {
        Piece<DT> x;
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x.w[0]), "=r"(x.w[1]), "=r"(x.w[2]), "=r"(x.w[3]) : "r"(slot) : "memory");
        return x;
    };
    // f of the thread's pieces of a chunk, one after another
    auto each = [&](auto f) {
        if constexpr (GRAD) {
            uint32_t slot = slots;
            #pragma unroll 4
            for (uint32_t i = 0; i < all; ++i, slot += kStride) f(piece(slot));
        } else {
            #pragma unroll
            for (uint32_t i = 0; i < kHeld; ++i) {
                if (i >= all) break;
                held[i].forget();
                f(held[i]);
            }
        }
    };
    load(v0);
    const int32_t id0 = present(tid, far0, z0);
    if (id0 >= 0) s0 = ds_load<DT>(src, (uint64_t)id0);

    const Two scales = two(p.scale, p.scale), scales1 = two(p.scale1, p.scale1);
    float m = kDsLowest;
    Two sums = two(0.0f, 0.0f), sums1 = sums;           // of the even and of the odd columns
    for (uint32_t v = v0;;) {
        float c = m;
        if constexpr (GRAD) asm volatile("cp.async.wait_all;" ::: "memory");
        each([&](const Piece<DT> &x) { c = x.max_with(c); });
        const float f = exp2_approx((m - c) * p.scale);
        sums = sums * two(f, f);
        if constexpr (DUAL) {
            const float f1 = exp2_approx((m - c) * p.scale1);
            sums1 = sums1 * two(f1, f1);
        }
        m = c;
        const Two from = two(-c, -c);
        each([&](const Piece<DT> &x) {
            Two a, a1;
            #pragma unroll
            for (int k = 0; k < kVals / 2; ++k) {
                const Two t = x.pair(k) + from, e = exp2_approx(t * scales);
                a = k == 0 ? e : a + e;
                if constexpr (DUAL) {
                    const Two e1 = exp2_approx(t * scales1);
                    a1 = k == 0 ? e1 : a1 + e1;
                }
            }
            sums = sums + a;
            if constexpr (DUAL) sums1 = sums1 + a1;
        });
        v += THREADS * p.vecs;
        if (v >= v1) break;
        load(v);
    }

    float sum, sum1 = 0.0f;
    {
        float odd;
        apart(sums, sum, odd);
        sum += odd;
        if constexpr (DUAL) { apart(sums1, sum1, odd); sum1 += odd; }
    }

    // the entries
    TeacherSums z = {kDsLowest, kDsLowest, 0.0f, 0.0f};
    bool some = false;
    auto enter = [&](uint32_t j, int32_t at, float zj, float sj) {
        if (j < entries) { id[j] = at; ze[j] = zj; se[j] = sj; }
        if (at < 0 || j == p.top) return;
        some = true;
        z.add(zj, sj, p.scale);
        if constexpr (GRAD) {
            uint32_t h = ((uint32_t)at * 2654435761u) & (p.table - 1);
            for (;;) {                                  // ends: the table has more slots than there are entries
                const uint32_t old = atomicCAS(&table[h], 0u, (uint32_t)at + 1u) & 0x7fffffffu;
                if (old == 0u) break;
                if (old == (uint32_t)at + 1u) { atomicOr(&table[h], 0x80000000u); break; }
                h = (h + 1) & (p.table - 1);
            }
        }
    };
    const bool entered = warp * 32 < entries;           // warps with entries: only they need what is known of them
    if (entered) {
        enter(tid, id0, z0, s0);
        for (uint32_t j = tid + THREADS; j < entries; j += THREADS) {
            float zj = 0.0f;
            const int32_t at = present(j, place_of(j, zj), zj);
            enter(j, at, zj, at >= 0 ? ds_load<DT>(src, (uint64_t)at) : 0.0f);
        }
        __syncwarp();
        z.template join<32>(p.scale);
    }
    {
        const float c = warp_max(m);
        sum = lanes_sum<32>(sum * exp2_approx((m - c) * p.scale));
        if constexpr (DUAL) sum1 = lanes_sum<32>(sum1 * exp2_approx((m - c) * p.scale1));
        m = c;
    }
    if constexpr (kWarps > 1) {
        if (lane == 0) {
            parts[0][warp] = m; parts[1][warp] = sum; parts[2][warp] = sum1;
            parts[3][warp] = z.zm; parts[4][warp] = z.sm; parts[5][warp] = z.sum; parts[6][warp] = z.dot;
        }
        some = __syncthreads_or(some);
        const uint32_t from = lane % kWarps;
        const float c = parts[0][from];
        m = warp_max(c);
        sum = lanes_sum<kWarps>(parts[1][from] * exp2_approx((c - m) * p.scale));
        if constexpr (DUAL) sum1 = lanes_sum<kWarps>(parts[2][from] * exp2_approx((c - m) * p.scale1));
        if (entered) {
            z = {parts[3][from], parts[4][from], parts[5][from], parts[6][from]};
            z.template join<kWarps>(p.scale);
        }
    } else some = __any_sync(0xffffffffu, some);
    if (nrank > 1) {
        const uint32_t at = smem_u32(joint);
        if (tid == 0) { joint[0] = m; joint[1] = sum; joint[2] = sum1; }
        // Only the first warp's arrival has something to release; a release costs a warp about a tenth of its time here.
        __syncwarp();
        if (warp == 0) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        const uint32_t from = lane % nrank;             // 2, 4 or 8
        const float m0 = shared_of(at, from);
        sum = shared_of(at + 4, from);
        if constexpr (DUAL) sum1 = shared_of(at + 8, from);
        m = warp_max(m0);
        sum *= exp2_approx((m0 - m) * p.scale);
        if constexpr (DUAL) sum1 *= exp2_approx((m0 - m) * p.scale1);
        for (uint32_t d = nrank / 2; d > 0; d >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if constexpr (DUAL) sum1 += __shfl_xor_sync(0xffffffffu, sum1, d);
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");           // what was read has been used; waited for at the end
    }
    const int32_t label = id[p.top];
    if (rank == 0 && tid == 0) {
        const float s1 = DUAL ? sum1 : sum;             // the label's sum
        float loss = 0.0f;
        if (some) loss = p.alpha * p.temperature * (z.dot / z.sum + (m - z.sm) + p.temperature * (logf(sum) - logf(z.sum)));
        if (label >= 0) loss += p.beta * (logf(s1) - (se[p.top] - m));
        p.loss[row] = loss;
    }

    if constexpr (GRAD) {
        const float kt = some ? w * p.alpha * p.temperature : 0.0f, k1 = label >= 0 ? w * p.beta : 0.0f;
        const bool dead = !some && label < 0;           // zeros, whatever the logits are
        const float ct = DUAL ? kt / sum : (kt + k1) / sum, c1 = DUAL ? k1 / sum1 : 0.0f;
        auto slope = [&](float s) {
            const float t = s - m;
            float d = exp2_approx(t * p.scale) * ct;
            if constexpr (DUAL) d += exp2_approx(t * p.scale1) * c1;
            return d;
        };
        const Two from = two(-m, -m), cts = two(ct, ct), c1s = two(c1, c1);
        auto slopes = [&](uint32_t slot) {
            const Piece<DT> x = piece(slot);
            uint32_t q[4];
            #pragma unroll
            for (int k = 0; k < kVals / 2; ++k) {
                const Two t = x.pair(k) + from;
                Two d = exp2_approx(t * scales) * cts;
                if constexpr (DUAL) d = fma(DT == LGN_BF16 && k != 0 ? exp2_poly(t * scales1) : exp2_approx(t * scales1), c1s, d);
                float lo, hi;
                apart(d, lo, hi);
                if constexpr (DT == LGN_F32) { q[2 * k] = __float_as_uint(lo); q[2 * k + 1] = __float_as_uint(hi); }
                else q[k] = pack_bf16(lo, hi);
            }
            return make_uint4(q[0], q[1], q[2], q[3]);
        };
        const bool held = v1 - v0 <= THREADS * p.vecs; // the one chunk is still there
        auto write = [&](auto f) {
            for (uint32_t v = v0; v < v1; v += THREADS * p.vecs) {
                if (!held) {
                    load(v);
                    asm volatile("cp.async.wait_all;" ::: "memory");
                }
                if (!alike) whole = skip = all;             // a gradient that is aligned differently from its logits
                char *to = dst - shift * ES + (uint64_t)(v + tid) * 16 + skip * kStride;
                uint32_t slot = slots + skip * kStride;
                #pragma unroll 2
                for (uint32_t i = skip; i < whole; ++i, slot += kStride, to += kStride) {
                    const uint4 q = f(slot);
                    asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" :: "l"(to), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
                }
                #pragma unroll 1
                for (uint32_t i = 0; i < all; ++i) {
                    if (i >= skip && i < whole) i = whole;
                    if (i < all) store_edge<DT>(dst, (int64_t)(v + i * THREADS + tid) * kVals - shift, p.vocab, f(slots + i * kStride));
                }
            }
        };
        if (dead) write([](uint32_t) { return make_uint4(0u, 0u, 0u, 0u); });
        else write(slopes);
        __syncthreads();                                // the places are written over what other threads wrote there
        const int64_t begin = (int64_t)v0 * kVals - shift, end = (int64_t)v1 * kVals - shift;
        for (uint32_t j = tid; j < entries; j += THREADS) {
            const int32_t at = id[j];
            if (at < 0 || at < begin || at >= end) continue;
            uint32_t h = ((uint32_t)at * 2654435761u) & (p.table - 1), slot;
            while (((slot = table[h]) & 0x7fffffffu) != (uint32_t)at + 1u && slot != 0u) h = (h + 1) & (p.table - 1);
            float d = slope(se[j]);
            if (j < p.top) {
                float pt = exp2_approx((ze[j] - z.zm) * p.scale);
                if (slot >> 31) {
                    pt = 0.0f;
                    for (uint32_t i = 0; i < p.top; ++i) if (id[i] == at) pt += exp2_approx((ze[i] - z.zm) * p.scale);
                }
                d -= kt * (pt / z.sum);
                if (at == label) d -= k1;
            } else {
                if (slot != 0u) continue;               // an entry has the label's place
                d -= k1;
            }
            ds_store<DT>(dst, (uint64_t)at, d);
        }
    }
    __syncwarp();
    if (nrank > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // the other ranks have read this one's sums
}

#define LGN_DS(D, T, U, G) reinterpret_cast<const void *>(&distill_kernel<D, T, U, G>)
#define LGN_DS4(D, T, L) {{LGN_DS(D, L, false, false), LGN_DS(D, T, false, true)}, {LGN_DS(D, L, true, false), LGN_DS(D, T, true, true)}}
static const void *const kDistillTable[2][3][2][2] = {{LGN_DS4(LGN_F32, 32, 32), LGN_DS4(LGN_F32, 64, 64), LGN_DS4(LGN_F32, 128, 256)},
                                                      {LGN_DS4(LGN_BF16, 32, 32), LGN_DS4(LGN_BF16, 64, 64), LGN_DS4(LGN_BF16, 128, 256)}};
#undef LGN_DS4
#undef LGN_DS

}  // namespace lgn

using namespace lgn;

extern "C" lgn_status lgn_distill_loss(const void *logits, uint64_t tokens, uint64_t vocab, uint64_t ld, lgn_dtype dt,
                                       const void *ids, int ids_bits, uint64_t ld_ids, const void *teacher, uint64_t ld_teacher,
                                       lgn_dtype teacher_dt, uint64_t top, const void *labels, int label_bits,
                                       double temperature, double alpha, const float *weight,
                                       float *loss, void *dlogits, uint64_t ld_dlogits, void *stream) {
    if ((dt != LGN_F32 && dt != LGN_BF16) || (teacher_dt != LGN_F32 && teacher_dt != LGN_BF16)) return LGN_ERR_INVALID_ARG;
    if ((ids_bits != 32 && ids_bits != 64) || (label_bits != 32 && label_bits != 64)) return LGN_ERR_INVALID_ARG;
    if (!(temperature >= 1e-3 && temperature <= 1e3) || !(alpha >= 0.0 && alpha <= 1.0)) return LGN_ERR_INVALID_ARG;
    if (tokens > kDsMaxDim || vocab > kDsMaxDim || top > kDsMaxTop) return LGN_ERR_UNSUPPORTED;
    if (tokens == 0) return LGN_OK;
    const uint64_t es = dt == LGN_F32 ? 4 : 2, tes = teacher_dt == LGN_F32 ? 4 : 2, ies = (uint64_t)ids_bits / 8, les = (uint64_t)label_bits / 8;
    if (loss == nullptr || !aligned_to(loss, 4) || !aligned_to(weight, 4) || !aligned_to(labels, les)) return LGN_ERR_INVALID_ARG;
    if (vocab > 0 && (logits == nullptr || !aligned_to(logits, es) || ld < vocab || ld > (1ull << 40))) return LGN_ERR_INVALID_ARG;
    if (top > 0 && (ids == nullptr || teacher == nullptr || !aligned_to(ids, ies) || !aligned_to(teacher, tes) || ld_ids < top || ld_teacher < top ||
                    ld_ids > (1ull << 40) || ld_teacher > (1ull << 40))) return LGN_ERR_INVALID_ARG;
    if (vocab > 0 && dlogits != nullptr && (!aligned_to(dlogits, es) || ld_dlogits < vocab || ld_dlogits > (1ull << 40))) return LGN_ERR_INVALID_ARG;
    const uint64_t lb = vocab > 0 ? matrix_bytes(tokens, vocab, ld, es) : 0, db = vocab > 0 && dlogits != nullptr ? matrix_bytes(tokens, vocab, ld_dlogits, es) : 0;
    const uint64_t ib = top > 0 ? matrix_bytes(tokens, top, ld_ids, ies) : 0, tb = top > 0 ? matrix_bytes(tokens, top, ld_teacher, tes) : 0;
    if (vocab > 0 && (lb == 0 || (dlogits != nullptr && db == 0))) return LGN_ERR_INVALID_ARG;
    if (top > 0 && (ib == 0 || tb == 0)) return LGN_ERR_INVALID_ARG;
    const uint64_t wb = weight != nullptr ? 4 * tokens : 0, yb = labels != nullptr ? les * tokens : 0;
    struct { const void *p; uint64_t n; } in[5] = {{logits, lb}, {ids, ib}, {teacher, tb}, {weight, wb}, {labels, yb}};
    const bool in_place = dlogits == logits && ld_dlogits == ld;        // rows are read before they are written
    for (int i = 0; i < 5; ++i) {
        if (ranges_overlap(loss, 4 * tokens, in[i].p, in[i].n)) return LGN_ERR_INVALID_ARG;
        if (!(i == 0 && in_place) && ranges_overlap(dlogits, db, in[i].p, in[i].n)) return LGN_ERR_INVALID_ARG;
    }
    if (ranges_overlap(loss, 4 * tokens, dlogits, db)) return LGN_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms < 1) return LGN_ERR_CUDA;

    DistillArgs p = {};
    p.logits = static_cast<const char *>(logits); p.dlogits = static_cast<char *>(dlogits);
    p.ids = ids; p.labels = labels; p.teacher = static_cast<const char *>(teacher); p.weight = weight; p.loss = loss;
    p.ld = ld; p.ldd = ld_dlogits; p.ld_ids = ld_ids; p.ld_teacher = ld_teacher;
    p.vocab = (uint32_t)vocab; p.top = (uint32_t)top;
    p.ids64 = ids_bits == 64; p.labels64 = label_bits == 64; p.teacher_dt = teacher_dt;
    p.temperature = (float)temperature; p.alpha = (float)alpha; p.beta = (float)(1.0 - alpha);
    const bool both = alpha > 0.0 && alpha < 1.0 && labels != nullptr, dual = both && temperature != 1.0;
    p.scale1 = kLog2e;
    p.scale = (float)((alpha == 0.0 ? 1.0 : 1.0 / temperature) * 1.4426950408889634);
    const bool grad = dlogits != nullptr;
    if (grad) for (p.table = 16; p.table < 2 * (top + 1); p.table *= 2) {}
    const bool aligned = aligned_to(logits, 16) && (ld * es) % 16 == 0;
    const uint64_t vals = 16 / es, pieces = (vocab + vals - 1 + (aligned ? 0 : vals - 1)) / vals;        // of a row that is aligned worst
    // A gradient needs the row twice: the fewest threads of 32, 64 and 128 that hold it, or up to 8 CTAs of 128 (16 pieces per thread: what a CTA does
    // once costs as much as 40 values of each thread).  A loss alone passes through it once: 256 threads from 1024 pieces on, in chunks (4096 x 131072 bf16: 178 us after other work, 166 back to back;
    // 128 threads took a tenth longer).  More CTAs per row where there are too few rows to fill the machine.
    const int kind = pieces <= 32 * kDsVecs && top <= 128 && tokens >= 8 * (uint64_t)sms ? 0 : pieces <= 64 * kDsVecs ? 1 : 2;
    const unsigned threads = kind == 0 ? 32 : kind == 1 ? 64 : grad ? 128 : 256;
    const uint64_t per_cta = (uint64_t)threads * kDsVecs;
    unsigned cluster = 1;
    while (cluster < 8 && ((grad && pieces > cluster * per_cta) || (tokens * cluster < (uint64_t)sms && pieces > cluster * per_cta / 4))) cluster *= 2;
    p.pieces = (uint32_t)((pieces + cluster - 1) / cluster);
    if (tokens * cluster > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    p.slots = (uint32_t)((3 * (top + 1) + p.table + 3) & ~3ull);
    p.vecs = (p.pieces + threads - 1) / threads;
    if (grad) {                                             // chunks of one size
        const uint32_t chunks = (p.vecs + kDsVecs - 1) / kDsVecs;
        if (chunks > 1) p.vecs = (p.vecs + chunks - 1) / chunks;
    } else if (p.vecs > kDsVecs / 2) p.vecs = kDsVecs / 2;  // full ones, whose loads need no checks (4096 x 50021 bf16 after other work: 88 us, 102 with chunks of one size)
    const size_t smem = 4 * p.slots + (grad ? 16 * (size_t)threads * p.vecs : 0);
    log_line("distill_loss: tokens %llu vocab %llu top %llu, %s, %d threads, %u CTAs per row%s", (unsigned long long)tokens, (unsigned long long)vocab,
             (unsigned long long)top, dual ? "two softmaxes" : "one softmax", (int)threads, cluster, grad ? ", gradient" : "");
    const void *fn = kDistillTable[dt][kind][dual][grad];
    // Many entries.  The limit that holds without asking, 48 KB, covers the kernel's own variables too.  The same limit from every call: calls of two
    // threads must not lower one another's.
    if (smem + kDsStatic > 48 * 1024 && cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kDsMaxSmem) != cudaSuccess) {
        (void)cudaGetLastError();
        return LGN_ERR_CUDA;
    }
    void *args[] = {&p};
    return launch_dependent(fn, dim3((unsigned)(tokens * cluster)), dim3(threads), args, smem, stream, cluster);
}
