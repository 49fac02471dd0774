// Loss of a student's logits s against a teacher's top logits z at places id, and its gradient, row by row:
//
//   p = softmax(z / T) over the places present,   q = softmax(s / T),   q1 = softmax(s)
//   loss = a T^2 sum p (ln p - ln q[id]) + (1 - a) (-ln q1[label])
//   ds   = w (a T (q - p at id) + (1 - a) (q1 - 1 at label))
//
// With M = max s, S = sum exp((s - M) / T) and Z, zm the same of the teacher, the first part is
//   a T (1/Z sum exp((z - zm) / T) ((z - zm) - (s[id] - M))) + a T^2 (ln S - ln Z),
// so a row needs one pass for M and the sums and, for the gradient, one more over values that are still
// in registers: a CTA of 128 or 256 threads holds 8 x 16 bytes of a row per thread, and a cluster of up to 8 of them a row
// (their sums are joined through distributed shared memory).  Rows beyond that go through in chunks
// that are read again for the gradient, from L2 mostly.
//
// exp is taken in base 2 of (s - M) log2(e) / T, the difference first: it is exact or small where the term
// counts.  Sums are fp32, a few dozen terms per thread, then by lanes, warps and ranks in a fixed order.
//
// The gradient's places are written last, over what the pass wrote there.  A place named more than once
// (by entries, or an entry and the label) is found by a table of the ids in shared memory, and then summed in the order of the
// entries by every entry that names it, so that all of them write the same value.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "lgn.h"
#include "lgn_launch.h"
#include "lgn_log.h"
#include "lgn_tensor.cuh"
#include "lgn_values.cuh"

namespace lgn {

constexpr uint64_t kDsMaxTop = 1024, kDsMaxDim = 1ull << 30;
constexpr int kDsVecs = 8;                              // pieces of 16 bytes a thread holds
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
    int32_t ids64, labels64, teacher_dt;
    float temperature, alpha, beta;                     // beta = 1 - alpha
    float scale, scale1;                                // log2(e) / T and log2(e); the first alone where one softmax serves
};

__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
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

__device__ __forceinline__ float warp_max(float v) {
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
    #pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float shared_of(uint32_t addr, uint32_t rank) {
    uint32_t at;
    float x;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
    return x;
}

// DUAL: the two parts take softmaxes of different temperatures.
template <int DT, int THREADS, bool DUAL, bool GRAD>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
distill_kernel(const DistillArgs p) {
    constexpr int kVals = Piece<DT>::kVals, ES = 16 / kVals, kWarps = THREADS / 32;
    extern __shared__ uint32_t dyn[];
    __shared__ float wmax[kWarps], wsum[kWarps], wsum1[kWarps], wtop[kWarps], wz[kWarps], wd[kWarps];
    __shared__ float joint[3];
    __shared__ uint32_t some_s;
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
    if (tid == 0) some_s = 0u;
    if constexpr (GRAD) for (uint32_t i = tid; i < p.table; i += THREADS) table[i] = 0u;
    __syncthreads();
    dep_wait();

    const char *src = p.logits + row * p.ld * ES;
    char *dst = GRAD ? p.dlogits + row * p.ldd * ES : nullptr;
    const int64_t shift = (int64_t)((reinterpret_cast<uintptr_t>(src) & 15) / ES), vocab = (int64_t)p.vocab;
    const bool whole = GRAD && ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0;
    const uint32_t total = (uint32_t)((shift + vocab + kVals - 1) / kVals);             // pieces of the row
    const uint32_t v0 = min(rank * p.pieces, total), v1 = min(v0 + p.pieces, total);
    const uint32_t in0 = shift > 0 ? 1u : 0u, in1 = min(v1, (uint32_t)((shift + vocab) / kVals));   // whole pieces
    const char *base = src - shift * ES;
    constexpr uint32_t kNone = DT == LGN_F32 ? 0xff800000u : 0xff80ff80u;               // -inf

    // the row's first chunk is under way while the entries are looked at
    Piece<DT> x[kDsVecs];
    auto load = [&](uint32_t v) {
        #pragma unroll
        for (int i = 0; i < kDsVecs; ++i) {
            const uint32_t u = v + i * THREADS + tid;
            uint32_t (&w)[4] = x[i].w;
            if (u >= in0 && u < in1)
                asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(base + (uint64_t)u * 16) : "memory");
            else {
                const uint4 q = u < v1 ? load_edge<DT>(src, (int64_t)u * kVals - shift, p.vocab) : make_uint4(kNone, kNone, kNone, kNone);
                w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
            }
        }
    };
    load(v0);

    float top_max = kDsLowest;
    bool some = false;
    for (uint32_t j = tid; j < entries; j += THREADS) {
        int64_t at = -1;
        float z = 0.0f, s = 0.0f;
        if (j < p.top) {
            at = ds_id(p.ids, p.ids64, row * p.ld_ids + j);
            z = p.teacher_dt == LGN_F32 ? ds_load<LGN_F32>(p.teacher, row * p.ld_teacher + j) : ds_load<LGN_BF16>(p.teacher, row * p.ld_teacher + j);
            if (at < 0 || at >= vocab || z == -INFINITY || p.alpha == 0.0f) at = -1;
            else { some = true; top_max = fmaxf(top_max, z); }
        } else if (p.labels != nullptr && p.beta != 0.0f) {
            at = ds_id(p.labels, p.labels64, row);
            if (at < 0 || at >= vocab) at = -1;
        }
        if (at >= 0) {
            s = ds_load<DT>(src, (uint64_t)at);
            if constexpr (GRAD) {
                uint32_t h = ((uint32_t)at * 2654435761u) & (p.table - 1);
                for (;;) {                              // ends: the table has more slots than there are entries
                    const uint32_t old = atomicCAS(&table[h], 0u, (uint32_t)at + 1u) & 0x7fffffffu;
                    if (old == 0u) break;
                    if (old == (uint32_t)at + 1u) { atomicOr(&table[h], 0x80000000u); break; }
                    h = (h + 1) & (p.table - 1);
                }
            }
        }
        id[j] = (int32_t)at; ze[j] = z; se[j] = s;
    }
    if (some) some_s = 1u;

    // M and the sums
    float m = kDsLowest, sum = 0.0f, sum1 = 0.0f;
    for (uint32_t v = v0;;) {
        float c = m;
        #pragma unroll
        for (int i = 0; i < kDsVecs; ++i) c = x[i].max_with(c);
        sum *= exp2_approx((m - c) * p.scale);
        if constexpr (DUAL) sum1 *= exp2_approx((m - c) * p.scale1);
        m = c;
        #pragma unroll
        for (int i = 0; i < kDsVecs; ++i) {
            float a = 0.0f, a1 = 0.0f;
            x[i].forget();
            #pragma unroll
            for (int k = 0; k < kVals; ++k) {
                const float t = x[i].at(k) - m;
                a += exp2_approx(t * p.scale);
                if constexpr (DUAL) a1 += exp2_approx(t * p.scale1);
            }
            sum += a;
            sum1 += a1;
        }
        v += THREADS * kDsVecs;
        if (v >= v1) break;
        load(v);
    }
    {
        const float c = warp_max(m);
        sum = warp_sum(sum * exp2_approx((m - c) * p.scale));
        if constexpr (DUAL) sum1 = warp_sum(sum1 * exp2_approx((m - c) * p.scale1));
        top_max = warp_max(top_max);
        if (lane == 0) { wmax[warp] = c; wsum[warp] = sum; if constexpr (DUAL) wsum1[warp] = sum1; wtop[warp] = top_max; }
    }
    __syncthreads();
    some = some_s != 0u;
    m = wmax[0]; top_max = wtop[0];
    #pragma unroll
    for (int w = 1; w < kWarps; ++w) { m = fmaxf(m, wmax[w]); top_max = fmaxf(top_max, wtop[w]); }
    sum = 0.0f; sum1 = 0.0f;
    #pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        sum += wsum[w] * exp2_approx((wmax[w] - m) * p.scale);
        if constexpr (DUAL) sum1 += wsum1[w] * exp2_approx((wmax[w] - m) * p.scale1);
    }
    if (nrank > 1) {
        const uint32_t at = smem_u32(joint);
        if (tid == 0) { joint[0] = m; joint[1] = sum; joint[2] = sum1; }
        cluster_sync();
        const float own = m;
        for (uint32_t r = 0; r < nrank; ++r) m = fmaxf(m, r == rank ? own : shared_of(at, r));
        sum = 0.0f; sum1 = 0.0f;
        for (uint32_t r = 0; r < nrank; ++r) {
            const float d = shared_of(at, r) - m;
            sum += shared_of(at + 4, r) * exp2_approx(d * p.scale);
            if constexpr (DUAL) sum1 += shared_of(at + 8, r) * exp2_approx(d * p.scale1);
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");           // waited for at the end
    }

    // the teacher's part
    float z_sum = 0.0f, z_dot = 0.0f;
    for (uint32_t j = tid; j < p.top; j += THREADS) {
        float e = 0.0f;
        if (id[j] >= 0) {
            const float z = ze[j] - top_max;
            e = exp2_approx(z * p.scale);
            z_sum += e;
            if (e != 0.0f) z_dot += e * (z - (se[j] - m));
        }
        ze[j] = e;
    }
    z_sum = warp_sum(z_sum);
    z_dot = warp_sum(z_dot);
    if (lane == 0) { wz[warp] = z_sum; wd[warp] = z_dot; }
    __syncthreads();
    z_sum = 0.0f; z_dot = 0.0f;
    #pragma unroll
    for (int w = 0; w < kWarps; ++w) { z_sum += wz[w]; z_dot += wd[w]; }
    const int32_t label = id[p.top];
    const float s1 = DUAL ? sum1 : sum;                 // the label's sum
    if (rank == 0 && tid == 0) {
        float loss = 0.0f;
        if (some) loss = p.alpha * p.temperature * (z_dot / z_sum + p.temperature * (logf(sum) - logf(z_sum)));
        if (label >= 0) loss += p.beta * (logf(s1) - (se[p.top] - m));
        p.loss[row] = loss;
    }

    if constexpr (GRAD) {
        const float w = p.weight != nullptr ? __uint_as_float(ldro_u32(p.weight + row)) : 1.0f;
        const float kt = some ? w * p.alpha * p.temperature : 0.0f, k1 = label >= 0 ? w * p.beta : 0.0f;
        const bool dead = !some && label < 0;           // zeros, whatever the logits are
        const float ct = DUAL ? kt / sum : (kt + k1) / sum, c1 = DUAL ? k1 / sum1 : 0.0f;
        auto slope = [&](float s) {
            const float t = s - m;
            float d = exp2_approx(t * p.scale) * ct;
            if constexpr (DUAL) d += exp2_approx(t * p.scale1) * c1;
            return d;
        };
        const bool held = v1 - v0 <= THREADS * kDsVecs;       // the one chunk is still in registers
        for (uint32_t v = v0; v < v1; v += THREADS * kDsVecs) {
            if (!held) load(v);
            #pragma unroll
            for (int i = 0; i < kDsVecs; ++i) {
                const uint32_t u = v + i * THREADS + tid;
                if (u < v1) {
                    float d[kVals];
                    uint32_t w[4];
                    x[i].forget();
                    #pragma unroll
                    for (int k = 0; k < kVals; ++k) d[k] = dead ? 0.0f : slope(x[i].at(k));
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if constexpr (DT == LGN_F32) w[k] = __float_as_uint(d[k]);
                        else w[k] = pack_bf16(d[2 * k], d[2 * k + 1]);
                    }
                    if (whole && u >= in0 && u < in1)
                        asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" :: "l"(dst - shift * ES + (uint64_t)u * 16), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    else store_edge<DT>(dst, (int64_t)u * kVals - shift, p.vocab, make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
        }
        __syncthreads();                                // the places are written over what other threads wrote there
        const int64_t c0 = (int64_t)v0 * kVals - shift, c1_ = (int64_t)v1 * kVals - shift;
        for (uint32_t j = tid; j < entries; j += THREADS) {
            const int32_t at = id[j];
            if (at < 0 || at < c0 || at >= c1_) continue;
            uint32_t h = ((uint32_t)at * 2654435761u) & (p.table - 1);
            while ((table[h] & 0x7fffffffu) != (uint32_t)at + 1u) h = (h + 1) & (p.table - 1);   // it is there
            float pt = j < p.top ? ze[j] : 0.0f;
            if (table[h] >> 31) {
                pt = 0.0f;
                for (uint32_t i = 0; i < p.top; ++i) if (id[i] == at) pt += ze[i];
            }
            float d = slope(se[j]);
            if (some) d -= kt * (pt / z_sum);
            if (at == label) d -= k1;
            ds_store<DT>(dst, (uint64_t)at, d);
        }
    }
    __syncwarp();
    if (nrank > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // the other ranks have read this one's sums
}

#define LGN_DS(D, T, U, G) reinterpret_cast<const void *>(&distill_kernel<D, T, U, G>)
#define LGN_DS4(D, T) {{LGN_DS(D, T, false, false), LGN_DS(D, T, false, true)}, {LGN_DS(D, T, true, false), LGN_DS(D, T, true, true)}}
static const void *const kDistillTable[2][2][2][2] = {{LGN_DS4(LGN_F32, 128), LGN_DS4(LGN_F32, 256)}, {LGN_DS4(LGN_BF16, 128), LGN_DS4(LGN_BF16, 256)}};
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
    const uint64_t vals = 16 / es, pieces = (vocab + vals - 1 + vals - 1) / vals;        // however a row is aligned
    // 128 threads where they hold the row; else 256, and as many CTAs as hold it for a gradient.  More CTAs per row where there are
    // too few rows to fill the machine.
    const int big = pieces > 128 * kDsVecs;
    const uint64_t per_cta = (uint64_t)(big ? 256 : 128) * kDsVecs;
    unsigned cluster = 1;
    while (cluster < 8 && ((grad && pieces > cluster * per_cta) || (tokens * cluster < (uint64_t)sms && pieces > cluster * per_cta / 4))) cluster *= 2;
    p.pieces = (uint32_t)((pieces + cluster - 1) / cluster);
    if (tokens * cluster > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;
    const size_t smem = 4 * (3 * (top + 1) + p.table);
    log_line("distill_loss: tokens %llu vocab %llu top %llu, %s, %d threads, %u CTAs per row%s", (unsigned long long)tokens, (unsigned long long)vocab,
             (unsigned long long)top, dual ? "two softmaxes" : "one softmax", big ? 256 : 128, cluster, grad ? ", gradient" : "");
    void *args[] = {&p};
    return launch_dependent(kDistillTable[dt][big][dual][grad], dim3((unsigned)(tokens * cluster)), dim3(big ? 256 : 128), args, smem, stream, cluster);
}
