// Products of rows grouped by expert, on the tensor cores (tcgen05, TMA): the kernel and what its instances share with the host side.
//
// Rows of group e are start_e .. end_e - 1 of the activations, found on the device from the groups' offsets.
//   kGmRows  out[r, :] = X[r, :] W_e^T or X[r, :] W_e     tiles of 128 CTAS rows of one group by BN columns
//   kGmSwap  the same with the weights' 128 rows as the MMA's rows and BN activations as its columns: few rows per group;
//            the CTAs of a cluster take consecutive shares of k and add their tiles through distributed shared memory
//   kGmTurn  the same turned round for any number of rows: tiles of 128 CTAS weights' rows by up to BN activations, an MMA taking as many columns
//            as the tile has rows, in steps of 32, so that groups cost what their rows cost
//   kGmGrad  out_e = dY^T X over the rows of group e      tiles of 128 CTAS by BN of each group's matrix
//   kGmShare the same with each group's rows shared out over the CTAs of a cluster, as kGmSwap does: few tiles, long groups
// bf16 operands with fp32 sums, or 8-bit integers with 32-bit integer sums (exact) times a scale per row of either.
//
// A step of the contraction is 128 bytes of each row: 64 bf16 or 128 integers, four MMAs.  Operands whose rows run along
// the contraction lie in shared memory as rows of 128 bytes; the others (W in X W_e, both in the gradient) as
// boxes of 64 columns by 64 rows, which the MMA reads as they are (the descriptor's strides and the instruction's
// transpose bits say so), so that no operand is ever copied to another order.
//
// In the gradient the contraction runs over a group's rows, and its last step would reach into the next group.  The
// rows behind the group's end are written over with zeros in shared memory, up to the next multiple of 16, and the MMAs beyond
// are left out: a warp of its own (10) waits for that step's copies (on a barrier of each CTA), clears the rows
// and hands the step on, while the copies go on with the next tile's.  Nothing else sees rows of another group but the output rows that are not stored.
//
// Roles as in the 8-bit float product: warp 8 copies, warp 9 issues MMAs, warps 0..7 read sums out.  Sums of
// bf16 products leave tensor memory every 512 of the contraction for registers, because the tensor cores' additions
// truncate, here after every 16 products: sums of positive products come out too small by 9e-7 with 512, by twice that with 1024 and by 4e-7 with
// 256, which costs 2 to 4 % (16384 rows, 8 x 4096 x 4096: 393 us, 401).  Two accumulators take turns.  Every wait is bounded: that of the clearing
// warp, which has nothing to do until a group ends, from the last step that was copied in.
#pragma once

#include <type_traits>

#include "lgn.h"
#include "lgn_launch.h"
#include "lgn_tensor.cuh"

namespace lgn {

enum GmForm { kGmRows = 0, kGmSwap = 1, kGmGrad = 2, kGmShare = 3, kGmTurn = 4 };
enum GmKind { kGmBf16 = 0, kGmInt8 = 1 };

constexpr int kGmEpiWarps = 8;
constexpr int gm_threads(int form) { return form == kGmGrad || form == kGmShare ? 352 : 320; }
constexpr int kGmGroupRows = 16;                 // row tiles walked before the next column tile (L2 reuse)
constexpr uint32_t kGmChunk = 8;                 // steps whose sum stays in tensor memory (bf16)
constexpr int kGmBuffer = 4096;                  // 32 rows x 128 bytes of output

struct GmArgs {
    char *out;
    const void *offsets;                         // nullptr: one group of all rows
    const float *row_scales, *col_scales;        // of the activations; of the weights, group by group
    uint32_t *status;
    uint64_t ldo, out_group;                     // elements between rows, between groups' matrices (gradient)
    uint32_t rows, groups;                       // activations; experts
    uint32_t n;                                  // columns of the output
    uint32_t m;                                  // gradient: rows of each group's matrix
    uint32_t steps;                              // of the contraction (not in the gradient)
    uint32_t tiles_r, tiles_c;                   // column tiles; gradient: row tiles of a matrix
    uint32_t split_steps;                        // kGmSwap: steps of a CTA of a cluster
    uint32_t offsets64, accumulate, zero_rest, vec, withhold;
};

template <int KIND, int BN, int CTAS, int FORM> struct GmShape {
    static constexpr int kKeep = KIND == kGmInt8 ? 128 : 64;        // of the contraction in a step
    static constexpr int kStaging = FORM != kGmRows && FORM != kGmGrad ? 0 : kGmEpiWarps * kGmBuffer;
    static constexpr int kStageBytes = 128 * 128 + BN / CTAS * 128;
    static constexpr int kFit = ((FORM == kGmSwap ? 100 : 225) * 1024 - kStaging) / kStageBytes;
    static constexpr int kStages = kFit > 8 ? 8 : kFit;
    static constexpr int kSmem = 1024 + kStaging + kStages * kStageBytes;
    static constexpr int kTmemCols = 2 * BN;                        // a power of two from 32 on
    static_assert(kSmem <= 227 * 1024 && kTmemCols <= 512 && kTmemCols >= 32, "shapes");
    static constexpr int kPartPitch = 132;                          // floats between the rows of kGmShare's partial tile: no bank conflicts
    static_assert((FORM != kGmSwap || BN * 128 * 4 <= kStages * kStageBytes) && (FORM != kGmShare || (BN == 128 && CTAS == 1 && kPartPitch * 128 * 4 <= kStages * kStageBytes)),
                  "a partial tile takes the stages' place");
};

// ------------------------------------------------------------------ groups and tiles
struct GmTile { uint32_t group, start, end, r, c; };                // the group's rows; row tile within it, column tile

// A warp's walk over the tiles of all groups, in increasing order: lane l holds group base + l.
template <bool GRAD, int TILE_ROWS> struct GmWalk {
    const GmArgs &p;
    const uint32_t lane;
    uint32_t base, before, start, end, upto;                        // before: tiles ahead of the window; upto: through this lane's group

    __device__ __forceinline__ GmWalk(const GmArgs &args, uint32_t l) : p(args), lane(l) { open(0, p.offsets == nullptr ? 0 : at(0), 0); }

    // offset i, forced into the rows that there are
    __device__ __forceinline__ uint32_t at(uint32_t i) const {
        if (p.offsets64) {
            const int64_t v = (int64_t)ldro_u64(static_cast<const char *>(p.offsets) + 8 * (uint64_t)i);
            return v < 0 ? 0u : v > (int64_t)p.rows ? p.rows : (uint32_t)v;
        }
        const int32_t v = (int32_t)ldro_u32(static_cast<const char *>(p.offsets) + 4 * (uint64_t)i);
        return v < 0 ? 0u : min((uint32_t)v, p.rows);
    }
    // The window from group w on; `carry`: where it begins.  An offset below an earlier one counts as that one.
    __device__ __forceinline__ void open(uint32_t w, uint32_t carry, uint32_t tiles) {
        base = w;
        before = tiles;
        end = p.offsets == nullptr ? p.rows : w + lane < p.groups ? at(w + lane + 1) : 0u;
        end = max(end, carry);
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= (uint32_t)d) end = max(end, o);
        }
        start = __shfl_up_sync(0xffffffffu, end, 1);
        if (lane == 0) start = carry;
        upto = GRAD ? (w + lane < p.groups ? p.tiles_r * p.tiles_c : 0u) : (end - start + TILE_ROWS - 1) / TILE_ROWS * p.tiles_c;
        #pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= (uint32_t)d) upto += o;
        }
        upto += tiles;
    }
    __device__ __forceinline__ bool find(uint32_t t, GmTile &out) {
        for (;;) {
            const uint32_t total = __shfl_sync(0xffffffffu, upto, 31);
            if (t < total) break;
            if (p.groups - base <= 32) return false;
            open(base + 32, __shfl_sync(0xffffffffu, end, 31), total);
        }
        const uint32_t src = __ffs(__ballot_sync(0xffffffffu, upto > t)) - 1;
        const uint32_t prev = __shfl_sync(0xffffffffu, upto, src == 0 ? 0 : src - 1);
        out.group = base + src;
        out.start = __shfl_sync(0xffffffffu, start, src);
        out.end = __shfl_sync(0xffffffffu, end, src);
        const uint32_t in = t - (src == 0 ? before : prev);
        const uint32_t tr = GRAD ? p.tiles_r : (out.end - out.start + TILE_ROWS - 1) / TILE_ROWS;
        const uint32_t span = kGmGroupRows * p.tiles_c, g = in / span, rest = in % span, h = min((uint32_t)kGmGroupRows, tr - g * kGmGroupRows);
        out.r = g * kGmGroupRows + rest % h;
        out.c = rest / h;
        return true;
    }
    // Where the last group ends; the walk is over then.
    __device__ __forceinline__ uint32_t last() {
        GmTile t;
        while (find(0xffffffffu, t)) {}
        return __shfl_sync(0xffffffffu, end, 31);
    }
};

// ------------------------------------------------------------------ instructions
template <int CTAS>
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z) {
    if constexpr (CTAS == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// Boxes of 64 columns (128 bytes) by 64 rows, 128-byte swizzle: groups of 8 rows 1024 bytes apart, the next 64 columns 8192.
__device__ __forceinline__ uint64_t desc_boxes(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (512ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
template <int KIND, int CTAS>
__device__ __forceinline__ void mma_plain(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if constexpr (KIND == kGmInt8) {
        if constexpr (CTAS == 2)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
        else
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
    } else {
        if constexpr (CTAS == 2)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
        else
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
    }
}
// Arrival at the leader's barrier that releases this thread's shared-memory writes to it, and the wait that acquires them.
__device__ __forceinline__ void arrive_leader_release(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(in_leader(bar)) : "memory");
}
__device__ __forceinline__ bool mbar_try_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_warp_cluster(uint32_t bar, uint32_t parity, volatile uint32_t *stop) {
    if (!mbar_wait_warp(bar, parity, stop)) return false;
    return __all_sync(0xffffffffu, mbar_try_cluster(bar, parity));              // completed already: acquires for the cluster
}

// A wait that may begin long before what it is for: `steps` counts the steps that the copying warp has begun, and as long as it goes on counting the wait
// has its whole time.
static __device__ __noinline__ bool mbar_wait_behind_slow(uint32_t bar, uint32_t parity, volatile uint32_t *stop, volatile uint32_t *steps) {
    long long t0 = clock64();
    uint32_t seen = *steps;
    for (;;) {
        if (mbar_try(bar, parity)) return true;
        if (*stop) return false;
        const uint32_t now = *steps;
        if (now != seen) { seen = now; t0 = clock64(); }
        else if (clock64() - t0 > kMmWaitClocks) { *stop = 1u; return false; }
    }
}
__device__ __forceinline__ bool mbar_wait_warp_behind(uint32_t bar, uint32_t parity, volatile uint32_t *stop, volatile uint32_t *steps) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait_behind_slow(bar, parity, stop, steps));
}

// ------------------------------------------------------------------ output
// 32 rows x 128 bytes of the output from row y, column x of group z on; lane l holds row l in v, `valid` rows of the 32 are stored.  They are turned in
// the warp's staging buffer (128-byte swizzle) and leave as whole rows, 16 bytes a lane where rows are whole 16-byte pieces.  (TMA stores of the buffer
// instead had each buffer wait for its last copy: 2048 rows, 8 x 4096 x 4096 fp32, 200 us with one buffer per warp, 136 with two.)
template <int FORM, int ODT>
__device__ __forceinline__ void gm_store(const GmArgs &p, uint32_t buf, uint32_t y, uint32_t x, uint32_t z, uint32_t valid, uint32_t lane, float *v) {
    constexpr int kCols = OutRun<ODT>::kCols, kPer = kCols / 8, ES = 16 / kPer;
    char *out = p.out + ((FORM == kGmGrad ? (uint64_t)z * p.out_group : 0) + (uint64_t)y * p.ldo + x) * ES;
    if (FORM == kGmGrad && p.accumulate && lane < valid) {
        const char *row = out + lane * p.ldo * ES;
        #pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (p.vec) {
                if (x + (q + 1) * kPer <= p.n) {
                    uint32_t w[4];
                    ld128(row + q * 16, w);
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if constexpr (ODT == LGN_F32) v[4 * q + j] += __uint_as_float(w[j]);
                        else { v[8 * q + 2 * j] += __uint_as_float(w[j] << 16); v[8 * q + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u); }
                    }
                }
            } else {
                #pragma unroll
                for (int j = 0; j < kPer; ++j) if (x + q * kPer + j < p.n) v[q * kPer + j] += load_out<ODT>(row, q * kPer + j);
            }
        }
    }
    __syncwarp();                                           // the buffer's last contents have been read
    #pragma unroll
    for (int q = 0; q < 8; ++q) {
        uint32_t w[4];
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (ODT == LGN_F32) w[j] = __float_as_uint(v[4 * q + j]);
            else w[j] = pack_bf16(v[8 * q + 2 * j], v[8 * q + 2 * j + 1]);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};"
                     :: "r"(buf + lane * 128 + ((q ^ (lane & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
    __syncwarp();
    if (p.vec) {
        const uint32_t q = lane & 7;
        char *at = out + (uint64_t)(lane >> 3) * p.ldo * ES + q * 16;
        #pragma unroll 2                                    // more at once spills beside 128 sums (fp32, 16384 rows, 8 x 4096 x 4096: 470 us, 411)
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t r = 4 * i + (lane >> 3);
            if (r < valid && x + (q + 1) * kPer <= p.n) {
                uint32_t w[4];
                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(buf + r * 128 + ((q ^ (r & 7)) << 4)) : "memory");
                asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" :: "l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
            }
            at += 4 * p.ldo * ES;
        }
        return;
    }
    for (uint32_t r = 0; r < valid; ++r) {
        uint32_t w;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
        char *at = out + r * p.ldo * ES + lane * 4;
        if constexpr (ODT == LGN_F32) {
            if (x + lane < p.n) *reinterpret_cast<uint32_t *>(at) = w;
        } else {
            const uint32_t c = x + 2 * lane;
            if (c + 1 < p.n && (reinterpret_cast<uintptr_t>(at) & 3) == 0) *reinterpret_cast<uint32_t *>(at) = w;
            else {
                if (c < p.n) *reinterpret_cast<uint16_t *>(at) = (uint16_t)w;
                if (c + 1 < p.n) *reinterpret_cast<uint16_t *>(at + 2) = (uint16_t)(w >> 16);
            }
        }
    }
}

// Zeros for the rows ahead of the first and behind the last group, by all epilogue warps of the grid.
template <int ODT, class Walk>
__device__ __forceinline__ void gm_zero_rest(const GmArgs &p, Walk &walk, uint32_t warp, uint32_t lane) {
    if (!p.zero_rest || p.offsets == nullptr) return;
    const uint32_t head = walk.at(0), tail = walk.last(), count = head + (p.rows - tail);
    for (uint32_t i = blockIdx.x * kGmEpiWarps + warp; i < count; i += gridDim.x * kGmEpiWarps) {
        const uint64_t at = (uint64_t)(i < head ? i : tail + (i - head)) * p.ldo;
        for (uint32_t c = lane; c < p.n; c += 32) store_out<ODT>(p.out, at + c, 0.0f);
    }
}

// ------------------------------------------------------------------ the kernel
template <int KIND, int BN, int CTAS, int FORM, bool W_ALONG, int ODT>       // W_ALONG: the weights' rows run along the contraction
__global__ void __launch_bounds__(gm_threads(FORM), FORM == kGmSwap ? 2 : 1)
grouped_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const GmArgs p) {
    using S = GmShape<KIND, BN, CTAS, FORM>;
    constexpr bool kGrad = FORM == kGmGrad || FORM == kGmShare, kOne = FORM == kGmSwap || FORM == kGmShare;      // kOne: one tile per cluster
    constexpr bool kTurned = FORM == kGmSwap || FORM == kGmTurn;            // the weights are the MMA's rows
    using Walk = GmWalk<kGrad, kTurned ? BN : 128 * CTAS>;
    constexpr bool kBoxesA = kGrad || (kTurned && !W_ALONG), kBoxesB = kGrad || (FORM == kGmRows && !W_ALONG);
    constexpr int kPart = BN / CTAS;                        // columns that this CTA brings
    static_assert(!kBoxesB || kPart % 64 == 0, "boxes");
    constexpr int kRun = FORM == kGmSwap ? BN / 2 : FORM == kGmTurn ? 16 : FORM == kGmShare ? 32 : OutRun<ODT>::kCols;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[4 * S::kStages + 2 * 2 + 1];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t stop, begun;               // begun: steps whose copies warp 8 has issued (gradient)
    dep_launch();

    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u, staging0 = smem0 + S::kStages * S::kStageBytes, bar0 = smem_u32(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (S::kStages + s); };
    auto acc_full = [&](uint32_t a) { return bar0 + 8 * (2 * S::kStages + a); };
    auto acc_empty = [&](uint32_t a) { return bar0 + 8 * (2 * S::kStages + 2 + a); };
    const uint32_t drained = bar0 + 8 * (2 * S::kStages + 4);
    auto last_in = [&](uint32_t s) { return drained + 8 + 8 * s; };             // a group's last step is there, in this CTA
    auto peer_clear = [&](uint32_t s) { return drained + 8 + 8 * (S::kStages + s); };           // and cleared in the other

    uint32_t rank = 0, nrank = 1;                           // within the cluster: a pair, or the CTAs that share k
    if constexpr (CTAS == 2 || kOne) {
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(nrank));
    }
    const bool leader = CTAS == 1 || rank == 0;
    const uint32_t half = CTAS == 2 ? rank : 0;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint32_t tile0 = blockIdx.x / CTAS, tile_step = gridDim.x / CTAS;
    if constexpr (kOne) {                                   // one tile per cluster; more clusters than tiles are launched, the number being known here only
        tile0 = blockIdx.x / nrank;
        tile_step = 0x7fffffffu;
        dep_wait();
        Walk walk(p, lane);
        GmTile t;
        if (!walk.find(tile0, t)) {                         // the same for all CTAs of the cluster
            if (FORM == kGmSwap && warp < kGmEpiWarps) gm_zero_rest<ODT>(p, walk, warp, lane);
            return;
        }
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); mbar_init(last_in(s), 1); mbar_init(peer_clear(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), CTAS * kGmEpiWarps); }
        mbar_init(drained, 1);
        stop = 0u;
        begun = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        if constexpr (CTAS == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_base_s)), "n"(S::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_base_s)), "n"(S::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    fence_before();
    __syncthreads();
    if constexpr (CTAS == 2) cluster_sync();                // barriers of both CTAs are set up, tensor memory of both allocated
    fence_after();
    const uint32_t tmem = tmem_base_s;
    uint32_t k0 = 0, k1 = p.steps;                          // this CTA's steps, where they do not depend on the group
    if constexpr (FORM == kGmSwap) { k0 = min(p.steps, rank * p.split_steps); k1 = min(p.steps, k0 + p.split_steps); }
    auto steps_of = [&](const GmTile &t) {
        if constexpr (FORM == kGmShare) {
            const uint32_t all = (t.end - t.start + 63) / 64, each = (all + nrank - 1) / nrank;
            k0 = min(all, rank * each);
            return min(all, k0 + each) - k0;
        } else return kGrad ? (t.end - t.start + 63) / 64 : k1 - k0;
    };
    constexpr uint32_t kChunk = KIND == kGmInt8 ? 0x40000000u : kGmChunk;

    // kGmTurn: a group's rows in tiles of the same height; the rows of one and the MMA's columns for them
    auto span = [&](const GmTile &t, uint32_t &row0, uint32_t &cols) {
        const uint32_t len = t.end - t.start, count = (len + BN - 1) / BN, height = ((len + count - 1) / count + 31) & ~31u;
        row0 = t.start + t.r * height;
        cols = (min(height, t.end - row0) + 31) & ~31u;
    };

    uint32_t issued = 0, last_mask = 0, last_ph = 0;        // stages filled so far; with a last step; phases of last_in (warp 8)
    auto ragged = [&](uint32_t left) { return kGrad && left < 64 && (left & 15) != 0; };        // rows to clear in a step with `left` rows to the group's end
    if (warp == 8) {
        dep_wait();
        Walk walk(p, lane);
        GmTile t;
        uint32_t s = 0, ph = 1;
        bool ok = true;
        for (uint32_t i = tile0; ok && walk.find(i, t); i += tile_step) {
            const uint32_t steps = steps_of(t);
            // first coordinates of the operands: along the tile, and the group where it is the map's third
            uint32_t row0 = t.start + t.r * BN, cols = BN;
            if constexpr (FORM == kGmTurn) span(t, row0, cols);
            const uint32_t boxes = (cols / CTAS + 31) / 32;                     // kGmTurn: of 32 rows
            const int at_a = FORM == kGmRows ? (int)(t.start + (t.r * CTAS + half) * 128) : (int)(((kTurned ? t.c : t.r) * CTAS + half) * 128);
            const int at_b = kTurned ? (int)(row0 + half * (cols / CTAS)) : (int)(t.c * BN + half * kPart);
            const int z_a = kTurned ? (int)t.group : 0, z_b = FORM == kGmRows ? (int)t.group : 0;
            for (uint32_t k = 0; k < steps; ++k) {
                if (!(ok = mbar_wait_warp(empty(s), ph, &stop))) break;
                const uint32_t a = smem0 + s * S::kStageBytes, b = a + 128 * 128;
                const uint32_t left = kGrad ? t.end - t.start - (k0 + k) * 64 : 64;
                const int kx = kGrad ? (int)(t.start + (k0 + k) * 64) : (int)((k0 + k) * S::kKeep);
                // copies to barrier `bar`
                auto copies = [&](auto group, uint32_t bar) {
                    constexpr int G = decltype(group)::value;
                    if constexpr (kBoxesA) {
                        if (!(p.withhold && issued == 0)) tma_box<G>(a, &map_a, bar, at_a, kx, z_a);
                        tma_box<G>(a + 8192, &map_a, bar, at_a + 64, kx, z_a);
                    } else if (!(p.withhold && issued == 0)) tma_box<G>(a, &map_a, bar, kx, at_a, z_a);
                    if constexpr (kBoxesB) {
                        #pragma unroll
                        for (int j = 0; j < kPart / 64; ++j) tma_box<G>(b + 8192 * j, &map_b, bar, at_b + 64 * j, kx, z_b);
                    } else if constexpr (FORM == kGmTurn) {
                        for (uint32_t j = 0; j < boxes; ++j) tma_box<G>(b + 4096 * j, &map_b, bar, kx, at_b + 32 * (int)j, z_b);
                    } else tma_box<G>(b, &map_b, bar, kx, at_b, z_b);
                };
                const bool last = ragged(left);
                if (elect_one()) {
                    if (!last) {
                        if (leader) mbar_expect(full(s), CTAS * (FORM == kGmTurn ? 128 * 128 + boxes * 4096 : S::kStageBytes));   // the bytes of both CTAs
                        copies(std::integral_constant<int, CTAS>{}, CTAS == 2 ? in_leader(full(s)) : full(s));
                    } else {
                        mbar_expect(last_in(s), S::kStageBytes);
                        copies(std::integral_constant<int, 1>{}, last_in(s));
                    }
                }
                last_mask = last ? last_mask | 1u << s : last_mask & ~(1u << s);
                if (last) last_ph ^= 1u << s;
                ++issued;
                if (kGrad && lane == 0) begun = issued;
                if (++s == S::kStages) { s = 0; ph ^= 1; }
            }
        }
    } else if (kGrad && warp == 10) {
        dep_wait();
        Walk walk(p, lane);
        GmTile t;
        uint32_t s = 0, in_ph = 0, peer_ph = 0;             // bit s: of the next phase of last_in(s), peer_clear(s)
        bool ok = true;
        for (uint32_t i = tile0; ok && walk.find(i, t); i += tile_step) {
            const uint32_t steps = steps_of(t);
            if (steps == 0) continue;
            const uint32_t left = t.end - t.start - (k0 + steps - 1) * 64, at = (s + steps - 1) % S::kStages;
            s = (s + steps) % S::kStages;
            if (!ragged(left)) continue;
            // All steps of the tile, and of tiles with nothing to clear, come first: seconds, where a group has 10^8 rows.
            if (!(ok = mbar_wait_warp_behind(last_in(at), in_ph >> at & 1, &stop, &begun))) break;
            in_ph ^= 1u << at;
            const uint32_t a = smem0 + at * S::kStageBytes, upper = (left + 15) & ~15u;
            for (uint32_t j = left * 8 + lane; j < upper * 8; j += 32) {                  // 16 bytes each, in every box
                #pragma unroll
                for (int q = 0; q < S::kStageBytes / 8192; ++q)
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" :: "r"(a + q * 8192 + j * 16), "r"(0u) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if constexpr (CTAS == 2) {
                if (!leader) { if (lane == 0) arrive_leader_release(peer_clear(at)); }
                else if (!(ok = mbar_wait_warp_cluster(peer_clear(at), peer_ph >> at & 1, &stop))) break;
                peer_ph ^= 1u << at;
            }
            if (leader && lane == 0) mbar_arrive(full(at));
        }
    } else if (warp == 9) {
        dep_wait();                                         // the limit of the waits below is for this kernel's work, not for what runs before it
        if (leader) {
            constexpr uint32_t kIdesc = (KIND == kGmInt8 ? 2u << 4 : 1u << 4) | (1u << 7) | (1u << 10) | ((kBoxesA ? 1u : 0u) << 15) | ((kBoxesB ? 1u : 0u) << 16) |
                                        ((FORM == kGmTurn ? 0u : (uint32_t)(BN >> 3)) << 17) | ((uint32_t)(128 * CTAS >> 4) << 24);
            constexpr uint32_t kNextA = kBoxesA ? 2048 >> 4 : 2, kNextB = kBoxesB ? 2048 >> 4 : 2;   // from one MMA of a step to the next
            Walk walk(p, lane);
            GmTile t;
            uint32_t s = 0, ph = 0, n = 0;                                      // n: accumulators begun
            bool ok = true;
            for (uint32_t i = tile0; ok && walk.find(i, t); i += tile_step) {
                const uint32_t steps = steps_of(t);
                uint32_t idesc = kIdesc;
                if constexpr (FORM == kGmTurn) {
                    uint32_t row0, cols;
                    span(t, row0, cols);
                    idesc |= (cols >> 3) << 17;
                }
                for (uint32_t c0 = 0; ok && c0 < steps; c0 += kChunk) {
                    const uint32_t c1 = min(steps, c0 + kChunk), acc = n & 1;
                    if (!(ok = mbar_wait_warp(acc_empty(acc), (n >> 1 & 1) ^ 1, &stop))) break;
                    fence_after();
                    for (uint32_t k = c0; k < c1; ++k) {
                        if (!(ok = mbar_wait_warp(full(s), ph, &stop))) break;
                        fence_after();
                        const uint32_t a = smem0 + s * S::kStageBytes;
                        const uint64_t da = kBoxesA ? desc_boxes(a) : desc_codes(a), db = kBoxesB ? desc_boxes(a + 128 * 128) : desc_codes(a + 128 * 128);
                        const uint32_t count = kGrad ? min(4u, (t.end - t.start - (k0 + k) * 64 + 15) / 16) : 4;
                        if (elect_one()) {
                            #pragma unroll
                            for (uint32_t j = 0; j < 4; ++j)
                                if (!kGrad || j < count)
                                    mma_plain<KIND, CTAS>(tmem + acc * BN, da + j * kNextA, db + j * kNextB, idesc, k > c0 || j > 0);
                            mma_commit<CTAS>(empty(s));
                            if (k + 1 == c1) mma_commit<CTAS>(acc_full(acc));
                        }
                        __syncwarp();
                        if (++s == S::kStages) { s = 0; ph ^= 1; }
                    }
                    ++n;
                }
            }
        }
    } else {
        dep_wait();                                                             // the output may belong to work before this call
        Walk walk(p, lane);
        GmTile t;
        uint32_t n = 0;
        const uint32_t quad = warp & 3, buf = staging0 + warp * kGmBuffer;
        bool ok = true;
        for (uint32_t i = tile0; ok && walk.find(i, t); i += tile_step) {
            const uint32_t steps = steps_of(t);
            uint32_t row0 = t.start + t.r * BN, part_cols = BN / 2;             // turned: the tile's first row; columns of this warp's part
            if constexpr (FORM == kGmTurn) { span(t, row0, part_cols); part_cols /= 2; }
            const uint32_t col0 = (warp >> 2) * part_cols, tmem_at = tmem + ((quad * 32u) << 16) + col0;
            const uint32_t y = (FORM == kGmRows ? t.start : 0) + ((kTurned ? t.c : t.r) * CTAS + half) * 128 + quad * 32;   // first of the warp's MMA rows
            const uint32_t y_end = FORM == kGmRows ? t.end : kGrad ? p.m : p.n, valid = y < y_end ? min(32u, y_end - y) : 0;
            float lane_scale = 0.0f;
            if constexpr (KIND == kGmInt8) {
                if (lane < valid) lane_scale = __uint_as_float(ldro_u32(kTurned ? p.col_scales + (uint64_t)t.group * p.n + y + lane : p.row_scales + y + lane));
            }
            // RUN finished columns of the tile, from column c of the warp's part on
            auto put = [&](uint32_t c, float *v) {
                const uint32_t in_tile = col0 + c;
                if constexpr (kTurned) {
                    if (FORM == kGmSwap && nrank > 1) {
                        float *part = reinterpret_cast<float *>(smem_raw + (smem0 - smem_u32(smem_raw)));
                        #pragma unroll
                        for (int j = 0; j < kRun; ++j) part[(in_tile + j) * 128 + quad * 32 + lane] = v[j];
                    } else if (lane < valid) {
                        const uint32_t row = row0 + in_tile;
                        char *at = p.out + ((uint64_t)row * p.ldo + y + lane) * (ODT == LGN_F32 ? 4 : 2);
                        #pragma unroll
                        for (int j = 0; j < kRun; ++j) {
                            if (row + j < t.end) store_out<ODT>(at, 0, v[j]);
                            at += p.ldo * (ODT == LGN_F32 ? 4 : 2);
                        }
                    }
                } else if constexpr (FORM == kGmShare) {
                    float4 *part = reinterpret_cast<float4 *>(smem_raw + (smem0 - smem_u32(smem_raw)) + ((quad * 32 + lane) * S::kPartPitch + in_tile) * 4);
                    #pragma unroll
                    for (int j = 0; j < kRun / 4; ++j) part[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                } else gm_store<FORM, ODT>(p, buf, y, t.c * BN + in_tile, t.group, valid, lane, v);
            };
            if constexpr (KIND == kGmInt8) {
                if (steps > 0) {
                    if (!(ok = mbar_wait_warp(acc_full(n & 1), n >> 1 & 1, &stop))) break;
                    fence_after();
                }
                #pragma unroll 1
                for (uint32_t c = 0; c < part_cols; c += kRun) {
                    float v[kRun];
                    #pragma unroll
                    for (int j = 0; j < kRun; ++j) v[j] = 0.0f;
                    __syncwarp();
                    if (steps > 0) {
                        #pragma unroll
                        for (int j = 0; j < kRun; j += 16) tmem_load16(tmem_at + (n & 1) * BN + c + j, v + j);
                        #pragma unroll
                        for (int j = 0; j < kRun; j += 16) tmem_load_wait16(v + j);
                    }
                    if (FORM != kGmSwap || nrank == 1) {
                        const uint32_t x = kTurned ? row0 + col0 + c : t.c * BN + col0 + c;
                        const uint32_t x_end = kTurned ? t.end : p.n;
                        const float *scales = kTurned ? p.row_scales : p.col_scales + (uint64_t)t.group * p.n;
                        #pragma unroll
                        for (int j0 = 0; j0 < kRun; j0 += 32) {
                            const float mine = lane < kRun - j0 && x + j0 + lane < x_end ? __uint_as_float(ldro_u32(scales + x + j0 + lane)) : 0.0f;
                            #pragma unroll
                            for (int j = j0; j < kRun && j < j0 + 32; ++j) {
                                const float other = __shfl_sync(0xffffffffu, mine, j - j0), q = (float)__float_as_int(v[j]);
                                v[j] = kTurned ? q * other * lane_scale : q * lane_scale * other;          // the activation's scale first, as everywhere
                            }
                        }
                    }
                    put(c, v);
                }
                if (steps > 0) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_leader<CTAS>(acc_empty(n & 1));
                    ++n;
                }
            } else {
                float sum[BN / 2];
                #pragma unroll
                for (int c = 0; c < BN / 2; ++c) sum[c] = 0.0f;
                for (uint32_t c0 = 0; c0 < steps; c0 += kChunk) {
                    if (!(ok = mbar_wait_warp(acc_full(n & 1), n >> 1 & 1, &stop))) break;
                    __syncwarp();
                    fence_after();
                    #pragma unroll
                    for (int c = 0; c < BN / 2; c += 16) {
                        if (FORM == kGmTurn && c >= (int)part_cols) break;
                        float v[16];
                        tmem_load16(tmem_at + (n & 1) * BN + c, v);
                        tmem_load_wait16(v);
                        #pragma unroll
                        for (int j = 0; j < 16; ++j) sum[c + j] += v[j];
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_leader<CTAS>(acc_empty(n & 1));
                    ++n;
                }
                if (!ok) break;
                #pragma unroll
                for (int c = 0; c < BN / 2; c += kRun) {
                    if (FORM == kGmTurn && c >= (int)part_cols) break;
                    put(c, sum + c);
                }
            }
        }
        __syncwarp();
        if (!kGrad && ok) gm_zero_rest<ODT>(p, walk, warp, lane);
    }
    __syncwarp();
    if constexpr (FORM == kGmSwap) {
        if (nrank > 1) {
            // every CTA's partial tile is in its own shared memory: column c is added over the ranks, in rank order, by the CTA c mod nrank
            cluster_sync();
            Walk walk(p, lane);
            GmTile t;
            if (walk.find(tile0, t) && threadIdx.x < kGmEpiWarps * 32) {
                const uint32_t at_row = threadIdx.x & 127, y = t.c * 128 + at_row, row0 = t.start + t.r * BN;
                if (y < p.n) {
                    const float scale = KIND == kGmInt8 ? __uint_as_float(ldro_u32(p.col_scales + (uint64_t)t.group * p.n + y)) : 0.0f;
                    for (uint32_t c = rank + (threadIdx.x >> 7) * nrank; c < (uint32_t)BN && row0 + c < t.end; c += 2 * nrank) {
                        float v = 0.0f;
                        int32_t whole = 0;
                        for (uint32_t q = 0; q < nrank; ++q) {
                            uint32_t at;
                            float x;
                            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem0 + (c * 128 + at_row) * 4), "r"(q));
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
                            if constexpr (KIND == kGmInt8) whole += __float_as_int(x); else v += x;
                        }
                        if constexpr (KIND == kGmInt8) v = (float)whole * __uint_as_float(ldro_u32(p.row_scales + row0 + c)) * scale;
                        store_out<ODT>(p.out, (uint64_t)(row0 + c) * p.ldo + y, v);
                    }
                }
            }
        }
    }
    if constexpr (FORM == kGmShare) {
        // the same, by rows: row r is added and stored by the CTA r mod nrank, four columns per lane
        cluster_sync();
        Walk walk(p, lane);
        GmTile t;
        if (walk.find(tile0, t) && warp < kGmEpiWarps) {
            const uint32_t x = t.c * 128 + 4 * lane;
            for (uint32_t r = rank + warp * nrank; r < 128 && t.r * 128 + r < p.m; r += kGmEpiWarps * nrank) {
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                for (uint32_t q = 0; q < nrank; ++q) {
                    uint32_t at;
                    float a[4];
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem0 + (r * S::kPartPitch + 4 * lane) * 4), "r"(q));
                    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]) : "r"(at) : "memory");
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] += a[j];
                }
                const uint64_t i = (uint64_t)t.group * p.out_group + (uint64_t)(t.r * 128 + r) * p.ldo + x;
                #pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p.accumulate && x + j < p.n) v[j] += load_out<ODT>(p.out, i + j);
                if (p.vec && x + 4 <= p.n) {
                    if constexpr (ODT == LGN_F32) *reinterpret_cast<float4 *>(p.out + i * 4) = make_float4(v[0], v[1], v[2], v[3]);
                    else *reinterpret_cast<uint2 *>(p.out + i * 2) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                } else {
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) if (x + j < p.n) store_out<ODT>(p.out, i + j, v[j]);
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    // a wait ran out, whichever role's: the MMAs and the copies in flight, of both CTAs, end first
    if (stop && warp == 9 && leader) {
        if (elect_one()) mma_commit<CTAS>(drained);
        __syncwarp();
        mbar_drain(drained, 0);
    }
    if (stop && warp == 8)
        for (uint32_t b = issued > (uint32_t)S::kStages ? issued - S::kStages : 0; b < issued; ++b) {
            const uint32_t s = b % S::kStages;
            if (last_mask >> s & 1) mbar_drain(last_in(s), last_ph >> s & 1 ^ 1);
            else if (leader) mbar_drain(full(s), (b / S::kStages) & 1);
        }
    if constexpr (CTAS == 2 || kOne) cluster_sync();                            // nothing of the other CTAs is in flight any more
    fence_after();
    if (threadIdx.x == 0 && stop && p.status != nullptr) *p.status = (uint32_t)LGN_ERR_TIMEOUT;
    if (warp == 9) {
        if constexpr (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(S::kTmemCols));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(S::kTmemCols));
    }
}

// ------------------------------------------------------------------ instances
struct GmKernel {
    const void *fn;
    int kind, form, along, odt, bn, ctas, smem;             // along: W_ALONG
};
template <int KIND, int BN, int CTAS, int FORM, bool ALONG, int ODT>
GmKernel gm_kernel() {
    return {reinterpret_cast<const void *>(&grouped_kernel<KIND, BN, CTAS, FORM, ALONG, ODT>), KIND, FORM, ALONG, ODT, BN, CTAS, GmShape<KIND, BN, CTAS, FORM>::kSmem};
}
struct GmKernels { const GmKernel *first; int count; };
GmKernels gm_forward_kernels();                             // X W_e^T, bf16
GmKernels gm_input_kernels();                               // X W_e, bf16
GmKernels gm_weight_kernels();                              // dY^T X, bf16
GmKernels gm_int8_kernels();                                // X W_e^T, 8-bit integers

}  // namespace lgn
