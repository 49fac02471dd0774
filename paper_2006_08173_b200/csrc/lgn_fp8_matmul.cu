// out[i, j] (+)= sum over k of A[i, k] B[j, k], A and B in 8-bit floating point with one power-of-two scale
// per row and block of 128 k (lgn_fp8_quantize).
//
// The tensor cores apply the scales: tcgen05.mma kind::mxf8f6f4 multiplies each group of 32 k by an E8M0
// factor per row of either operand, read from tensor memory; a block of 128 is four groups with the same
// byte.  Sums are fp32, in tensor memory over 1024 k and in registers beyond, and are rounded once, to the
// output's type.
//
// One CTA, or a pair of CTAs on two SMs (CTAS = 2), works on tiles of 128 CTAS rows of one operand ("rows") by BN rows of
// the other ("cols").  In a pair the CTA of rank 0 issues the MMAs of both (cta_group::2) and each CTA brings
// its own 128 rows and one half of the BN: at 256 x 256 a step of k (128) costs an SM 32 KiB of shared-memory writes
// for 512 clocks of MMA, where a lone CTA's 128 x 192 needs 1.7 times that per flop
// (8192 x 8192 x 4096: 258 -> 216 us when pairs came in).  Small products take lone CTAs, persistent over tiles, or (SPLIT) one tile
// per cluster with the CTAs of a cluster taking consecutive shares of k and adding their fp32 tiles through
// distributed shared memory in rank order.
//   warp 8  brings codes into a ring of shared-memory stages (TMA, 128-byte swizzle) and, every fourth step, the 512-byte
//           scale tiles of four blocks;
//   warp 9  one thread issues the scale copies into tensor memory and four MMAs (k = 32 each) per step and half (below).  (Scales
//           written to tensor memory by four warps of their own, tcgen05.st, came out 8 to 16 % slower.)
//   warps 0..7  add up the chunks of k from tensor memory (warp w: lanes 32 (w mod 4) on, columns of part w / 4), round
//               and store.
// SWAP: `rows` runs along the contiguous dimension of the output, so that the 32 lanes of a warp, which hold
// 32 rows, write contiguous memory whatever the alignment.
//
// The tensor cores' additions truncate, which biases a sum towards zero by about 2e-10 of its
// size per k (measured: 2.0e-7 at k = 1024, 1e-6 and more from 8192).  Every 1024 k the tile is therefore added to sums in
// registers (round to nearest) and a fresh one begun elsewhere in tensor memory; the error then stays below
// 5e-7 (k up to 16384).  Of bf16 outputs, 7e-5 are a neighbour of the rounded exact sum at 2048 x 2048 x 16384 (1e-5 with
// positive operands); with the sum in tensor memory over the whole of k it was 3e-4 (1e-3).
// Tiles of up to 192 columns have two accumulators, used in turn.  A tile of 256 would leave no columns for the scales
// with two; its MMAs are issued for two halves of 128 columns, whose chunks of k end 512 k apart, and three accumulators
// of 128 columns go round: while two collect, the third is read out.
//
// Every wait is bounded: one that runs out raises a flag on which all roles stop; the copies and MMAs in
// flight are waited for (bounded too), tensor memory is freed and the kernel ends with *status set.
#include <cuda.h>
#include <cuda_runtime.h>

#include <mutex>

#include "lgn.h"
#include "lgn_fp8.cuh"
#include "lgn_launch.h"
#include "lgn_log.h"
#include "lgn_tensor.cuh"

namespace lgn {

constexpr int kMmThreads = 320;                // warps 0..7: epilogue, 8: copies, 9: MMA
constexpr int kMmEpiThreads = 256, kMmEpiWarps = 8;
constexpr int kMmGroupRows = 16;                 // row tiles walked before the next column tile (L2 reuse)

struct MmArgs {
    void *out;
    uint64_t ldo;
    uint32_t *status;
    uint32_t rows, cols;                         // extents of the two operands
    uint32_t kblocks, groups;                    // ceil(k / 128), ceil(k / 512)
    uint32_t tiles_r, tiles_c;
    uint32_t fmt_rows, fmt_cols;
    uint32_t split_groups;                       // groups of four blocks per CTA of a cluster
    uint32_t accumulate;
    uint32_t withhold;                           // self-test: each CTA leaves out its first copy
};

constexpr uint32_t kMmChunk = 8;                 // steps of k (128 each) that stay in tensor memory

constexpr int kMmBuffer = 4096;                   // 32 rows x 128 bytes of output

// Bytes and stages per CTA.
template <int BN, int CTAS, int ODT> struct MmShape {
    static constexpr int kBuffers = ODT == LGN_F32 ? 2 : 1;         // output buffers of an epilogue warp
    static constexpr int kStaging = kMmEpiWarps * kBuffers * kMmBuffer;
    static constexpr int kColBlocks = BN <= 128 ? 1 : 2;            // 128-row scale tiles a column tile touches
    static constexpr int kStageBytes = 128 * 128 + BN / CTAS * 128;
    static constexpr int kScaleBytes = 512 * (1 + kColBlocks);
    static constexpr int kFit = (int)((225 * 1024 - kStaging) / (kStageBytes + kScaleBytes));
    static constexpr int kStages = kFit > 8 ? 8 : kFit;
    static constexpr int kHalves = BN == 256 ? 2 : 1;               // column parts of a tile with accumulators of their own
    static constexpr int kMmaN = BN / kHalves;                      // columns of an MMA and of an accumulator
    static constexpr int kAccs = kHalves + 1;                       // accumulators in tensor memory
    static constexpr int kBoxRows = kMmaN / CTAS;                   // rows of `cols` in a copy; a half's rows come from all CTAs of a tile
    static constexpr int kScaleCol = kAccs * kMmaN;                 // first tensor-memory column of the scales
    static constexpr int kScaleCols = 4 * (1 + kColBlocks);
    static constexpr int kScaleBufs = 4;
    static constexpr int kSmem = 1024 + kStaging + kStages * (kStageBytes + kScaleBytes);
    static_assert(kScaleCol + kScaleBufs * kScaleCols <= 512, "tensor memory");
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

template <int CTAS>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t add) {
    if constexpr (CTAS == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add) : "memory");
}
// A scale tile (512 bytes of shared memory, no swizzle, groups of 8 rows of 16 bytes 128 bytes apart) to four columns of
// tensor memory, the same in each quarter of the lanes; of both CTAs of a pair.
template <int CTAS>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t smem) {
    const uint64_t desc = (uint64_t)((smem & 0x3ffffu) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
    if constexpr (CTAS == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" :: "r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" :: "r"(taddr), "l"(desc) : "memory");
}
// A warp's 32 rows x 128 bytes of the output from row y, column x on; lane l holds row l in v.  They go through
// the warp's staging buffer (128-byte swizzle, so that the lanes' writes spread over all banks) and one TMA store,
// which leaves out what lies outside the matrix and runs on while the warp reads its next columns.
// The warp's BUFS buffers from bufs on are used in turn.
template <int ODT, int BUFS>
__device__ __forceinline__ void store_staged(const MmArgs &p, const CUtensorMap *map, uint32_t bufs, uint32_t &turn, uint32_t y, uint32_t x, uint32_t lane, float *v) {
    constexpr int kCols = OutRun<ODT>::kCols, kPer = kCols / 8;                         // elements per 16 bytes
    if (p.accumulate && y + lane < p.rows) {
        const uint64_t i = (uint64_t)(y + lane) * p.ldo + x;
        #pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (x + (q + 1) * kPer <= p.cols) {
                uint32_t w[4];
                ld128(static_cast<const char *>(p.out) + (i + q * kPer) * (16 / kPer), w);
                #pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (ODT == LGN_F32) v[4 * q + j] += __uint_as_float(w[j]);
                    else { v[8 * q + 2 * j] += __uint_as_float(w[j] << 16); v[8 * q + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u); }
                }
            }
        }
    }
    const uint32_t buf = bufs + (turn++ % BUFS) * kMmBuffer;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" :: "n"(BUFS - 1) : "memory");   // the buffer's last contents have been read
    __syncwarp();
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
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0 && x < p.cols && y < p.rows) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
                     :: "l"(map), "r"(buf), "r"(x), "r"(y) : "memory");
    }
    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");             // an empty group where nothing was stored
}

enum MmForm { kFormRows = 0, kFormSwap = 1, kFormSplit = 2 };

// N values `step` elements apart from element i on, of which the first `count` exist; eight at a time, so that few
// addresses and old values are live at once.
template <int ODT, int N>
__device__ __forceinline__ void store_strided(void *out, uint64_t i, uint64_t step, uint32_t count, float *v, bool accumulate) {
    #pragma unroll
    for (int k = 0; k < N; k += 8) {
        if (accumulate) {
            #pragma unroll
            for (int j = 0; j < 8; ++j) if (k + j < (int)count) v[k + j] += load_out<ODT>(out, i + j * step);
        }
        #pragma unroll
        for (int j = 0; j < 8; ++j) if (k + j < (int)count) store_out<ODT>(out, i + j * step, v[k + j]);
        i += 8 * step;
        asm volatile("" ::: "memory");
    }
}

__device__ __forceinline__ void tile_at(const MmArgs &p, uint32_t t, uint32_t &tr, uint32_t &tc) {
    const uint32_t span = kMmGroupRows * p.tiles_c, g = t / span, in = t % span;
    const uint32_t h = min((uint32_t)kMmGroupRows, p.tiles_r - g * kMmGroupRows);
    tr = g * kMmGroupRows + in % h;
    tc = in / h;
}

// An epilogue warp's part of one tile, kMmaN / 2 columns of each half from tmem_at on: adds the chunks of k up in registers as they are
// finished, hands RUN columns at a time to `put` (half, column within the part).  `steps`: of k; `n` counts accumulators;
// false: a wait ran out.
template <class S, int RUN, class Full, class Release, class Put>
__device__ __forceinline__ bool drain_tile(uint32_t tmem_at, uint32_t steps, uint32_t &n, volatile uint32_t *stop, Full acc_full, Release release, Put put) {
    constexpr int kCols = S::kMmaN / 2;
    static_assert(kCols % RUN == 0, "columns");
    float sum[S::kHalves][kCols];                           // from zero: copying the first chunk instead costs registers (spills, 4096^3 bf16 53 -> 58 us)
    #pragma unroll
    for (int h = 0; h < S::kHalves; ++h) {
        #pragma unroll
        for (int c = 0; c < kCols; ++c) sum[h][c] = 0.0f;
    }
    auto add = [&](float *to) {
        const uint32_t acc = n % S::kAccs;
        if (!mbar_wait_warp(acc_full(acc), (n / S::kAccs) & 1, stop)) return false;
        __syncwarp();                                      // after a `put` that lanes outside the output passed over, too
        fence_after();
        #pragma unroll
        for (int c = 0; c < kCols; c += 16) {
            float v[16];
            tmem_load16(tmem_at + acc * S::kMmaN + c, v);
            tmem_load_wait16(v);
            #pragma unroll
            for (int j = 0; j < 16; ++j) to[c + j] += v[j];
        }
        fence_before();
        release(acc);
        ++n;
        return true;
    };
    if constexpr (S::kHalves == 1) {
        for (uint32_t k = 0; k < steps; k += kMmChunk) if (!add(sum[0])) return false;
    } else {
        // in the order in which they end: after 4 steps the first of half 1, after 8 of half 0, and so on; both halves' last with the tile
        const uint32_t items = (steps + kMmChunk / 2 - 1) / (kMmChunk / 2) + 1;
        for (uint32_t j = 0; j < items; j += 2) {
            if (!add(sum[1])) return false;
            if (j + 1 < items && !add(sum[0])) return false;
        }
    }
    #pragma unroll
    for (int h = 0; h < S::kHalves; ++h) {
        #pragma unroll
        for (int c = 0; c < kCols; c += RUN) put(h, c, sum[h] + c);
    }
    return true;
}

template <int BN, int CTAS, int FORM, int ODT>
__global__ void __launch_bounds__(kMmThreads, 1)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap map_rows, const __grid_constant__ CUtensorMap map_cols, const __grid_constant__ CUtensorMap map_sc_rows,
                  const __grid_constant__ CUtensorMap map_sc_cols, const __grid_constant__ CUtensorMap map_out, const MmArgs p) {
    using S = MmShape<BN, CTAS, ODT>;
    constexpr int kRun = FORM == kFormRows ? OutRun<ODT>::kCols : 32;
    extern __shared__ uint8_t smem_raw[];
    dep_launch();
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 2 * S::kAccs + 1];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile uint32_t stop;

    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging0 = smem0 + S::kStages * S::kStageBytes, scales0 = staging0 + S::kStaging;
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (S::kStages + s); };
    auto acc_full = [&](uint32_t a) { return bar0 + 8 * (2 * S::kStages + a); };
    auto acc_empty = [&](uint32_t a) { return bar0 + 8 * (2 * S::kStages + S::kAccs + a); };
    const uint32_t drained = bar0 + 8 * (2 * S::kStages + 2 * S::kAccs);

    uint32_t rank = 0, nrank = 1;                           // within the cluster: a pair, or the CTAs that share k
    if constexpr (CTAS == 2 || FORM == kFormSplit) {
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(nrank));
    }
    const bool leader = CTAS == 1 || rank == 0;             // issues the MMAs; full and acc_empty are its barriers
    const uint32_t half = CTAS == 2 ? rank : 0;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int a = 0; a < S::kAccs; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), CTAS * kMmEpiWarps); }
        mbar_init(drained, 1);
        stop = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" :: "l"(&map_rows) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&map_cols) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&map_sc_rows) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&map_sc_cols) : "memory");
        if constexpr (FORM == kFormRows) asm volatile("prefetch.tensormap [%0];" :: "l"(&map_out) : "memory");
    }
    if (warp == 9) {
        if constexpr (CTAS == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_base_s)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_base_s)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    fence_before();
    __syncthreads();
    if constexpr (CTAS == 2) cluster_sync();                // barriers of both CTAs are set up, tensor memory of both allocated
    fence_after();
    const uint32_t tmem = 0;                                // where an allocation of all 512 columns begins

    // this CTA's tiles and steps of k
    uint32_t tile0 = blockIdx.x / CTAS, tile_step = gridDim.x / CTAS, kb0 = 0, kb1 = p.kblocks;
    if constexpr (FORM == kFormSplit) {
        tile0 = blockIdx.x / nrank;
        tile_step = 0x7fffffffu;
        kb0 = rank * p.split_groups * 4;
        kb1 = min(p.kblocks, kb0 + p.split_groups * 4);
    }
    const uint32_t tiles = p.tiles_r * p.tiles_c;

    // Warps 8 and 9 run their loops whole, one elected lane issuing: in code that only one lane runs the compiler moves every
    // operand of a TMA or MMA instruction to a uniform register at each use, which took 700 clocks per step of k.
    uint32_t issued = 0;                                    // stages filled so far (warp 8)
    if (warp == 8) {
        dep_wait();
        uint32_t s = 0, ph = 1, it = 0;
        bool ok = true;
        for (uint32_t t = tile0; ok && t < tiles; t += tile_step) {
            uint32_t tr, tc;
            tile_at(p, t, tr, tc);
            const int y_rows = (int)((tr * CTAS + half) * 128), y_cols = (int)(tc * BN + half * S::kBoxRows);
            int y_sr = (int)((tr * CTAS + half) * p.groups + (kb0 >> 2)), y_sc = (int)(((tc * BN) >> 7) * p.groups + (kb0 >> 2));
            for (uint32_t kb = kb0; kb < kb1; ++kb, ++it) {
                if (!(ok = mbar_wait_warp(empty(s), ph, &stop))) break;
                const uint32_t a = smem0 + s * S::kStageBytes, bar = CTAS == 2 ? in_leader(full(s)) : full(s);
                const bool with_scales = (kb & 3) == 0;
                if (elect_one()) {
                    if (leader) mbar_expect(full(s), CTAS * (S::kStageBytes + (with_scales ? S::kScaleBytes : 0)));   // the bytes of both CTAs
                    if (!(p.withhold != 0 && it == 0)) tma_tile<CTAS>(a, &map_rows, bar, (int)(kb * 128), y_rows);
                    #pragma unroll
                    for (int h = 0; h < S::kHalves; ++h)
                        tma_tile<CTAS>(a + (128 + h * S::kBoxRows) * 128, &map_cols, bar, (int)(kb * 128), y_cols + h * S::kMmaN);
                    if (with_scales) {                                          // tiles past the end read as zeros
                        const uint32_t sc = scales0 + s * S::kScaleBytes;
                        tma_tile<CTAS>(sc, &map_sc_rows, bar, 0, y_sr);
                        #pragma unroll
                        for (int b = 0; b < S::kColBlocks; ++b) tma_tile<CTAS>(sc + 512 * (1 + b), &map_sc_cols, bar, 0, y_sc + b * (int)p.groups);
                    }
                }
                if (with_scales) { ++y_sr; ++y_sc; }
                if (++s == S::kStages) { s = 0; ph ^= 1; }
            }
        }
        issued = it;
    } else if (warp == 9) {
        dep_wait();                                         // the limit of the waits below is for this kernel's work, not for what runs before it
        if (leader) {
            const uint32_t idesc0 = (p.fmt_rows << 7) | (p.fmt_cols << 10) | ((uint32_t)(S::kMmaN >> 3) << 17) | (1u << 23) | ((uint32_t)CTAS << 27);
            const uint64_t desc0 = desc_codes(smem0);
            constexpr uint32_t kTurn = kMmChunk / S::kHalves;                   // steps between two changes of accumulator
            uint32_t s = 0, ph = 0, n = 0, grp = 0;                             // n: accumulators begun
            bool ok = true;
            for (uint32_t t = tile0; ok && t < tiles; t += tile_step) {
                uint32_t tr, tc, sa = 0, acc[S::kHalves];
                tile_at(p, t, tr, tc);
                const uint32_t col_off = 4 + (((tc * BN) & 127) >> 5);          // columns' scales: the tile may begin inside a scale tile
                for (uint32_t c0 = kb0, turn = 0; ok && c0 < kb1; c0 += kTurn, ++turn) {
                    const uint32_t c1 = min(kb1, c0 + kTurn);
                    bool fresh[S::kHalves], ends[S::kHalves];                   // an accumulator begins, ends with this turn
                    #pragma unroll
                    for (int h = S::kHalves - 1; h >= 0; --h) {
                        // half 1 begins at turns 0 (for half a chunk), 1, 3, 5, half 0 at turns 0, 2, 4
                        fresh[h] = S::kHalves == 1 || turn == 0 || (turn & 1) == (uint32_t)h;
                        ends[h] = S::kHalves == 1 || c1 == kb1 || (turn & 1) != (uint32_t)h;
                        if (fresh[h]) {
                            acc[h] = n % S::kAccs;
                            ok = ok && mbar_wait_warp(acc_empty(acc[h]), (n / S::kAccs & 1) ^ 1, &stop);
                            ++n;
                        }
                    }
                    if (!ok) break;
                    fence_after();
                    for (uint32_t kb = c0; kb < c1; ++kb) {
                        if (!(ok = mbar_wait_warp(full(s), ph, &stop))) break;
                        fence_after();
                        const bool with_scales = (kb & 3) == 0;
                        if (with_scales) {
                            sa = tmem + S::kScaleCol + grp * S::kScaleCols;
                            grp = (grp + 1) % S::kScaleBufs;
                        }
                        const uint32_t idesc = idesc0 | ((kb & 3) << 4) | ((kb & 3) << 29);
                        const uint64_t da = desc0 + s * (uint32_t)(S::kStageBytes >> 4), db = da + (128 * 128 >> 4);
                        if (elect_one()) {
                            if (with_scales) {
                                #pragma unroll
                                for (int b = 0; b < 1 + S::kColBlocks; ++b) copy_scales<CTAS>(sa + 4 * b, scales0 + s * S::kScaleBytes + 512 * b);
                            }
                            #pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                #pragma unroll
                                for (int h = S::kHalves - 1; h >= 0; --h)
                                    mma_scaled<CTAS>(tmem + acc[h] * S::kMmaN, da + 2 * k, db + h * (S::kBoxRows * 128 >> 4) + 2 * k, idesc,
                                                     sa, sa + col_off + 4 * h, !fresh[h] || kb > c0 || k > 0);
                            }
                            mma_commit<CTAS>(empty(s));
                            if (kb + 1 == c1) {
                                #pragma unroll
                                for (int h = S::kHalves - 1; h >= 0; --h) if (ends[h]) mma_commit<CTAS>(acc_full(acc[h]));
                            }
                        }
                        __syncwarp();
                        if (++s == S::kStages) { s = 0; ph ^= 1; }
                    }
                }
            }
        }
    } else {
        dep_wait();                                                             // the output may belong to work before this call
        uint32_t n = 0, turn = 0;
        const uint32_t quad = warp & 3, col0 = (warp >> 2) * (S::kMmaN / 2), tmem_at = tmem + ((quad * 32u) << 16) + col0;
        for (uint32_t t = tile0; t < tiles; t += tile_step) {
            uint32_t tr, tc;
            tile_at(p, t, tr, tc);
            const uint32_t r = (tr * CTAS + half) * 128 + quad * 32 + lane;
            const bool ok = drain_tile<S, kRun>(tmem_at, kb1 - kb0, n, &stop, acc_full,
                [&](uint32_t acc) { __syncwarp(); if (lane == 0) arrive_leader<CTAS>(acc_empty(acc)); },
                [&](uint32_t h, uint32_t c, float *v) {
                    const uint32_t in_tile = h * S::kMmaN + col0 + c, x = tc * BN + in_tile;
                    if constexpr (FORM == kFormSplit) {
                        float *part = reinterpret_cast<float *>(smem_raw + (smem0 - smem_u32(smem_raw)));
                        #pragma unroll
                        for (int j = 0; j < 32; ++j) part[(in_tile + j) * 128 + quad * 32 + lane] = v[j];
                    } else if constexpr (FORM == kFormSwap) {
                        if (r < p.rows && x < p.cols)
                            store_strided<ODT, kRun>(p.out, (uint64_t)x * p.ldo + r, p.ldo, p.cols - x, v, p.accumulate != 0);
                    } else store_staged<ODT, S::kBuffers>(p, &map_out, staging0 + warp * (S::kBuffers * kMmBuffer), turn, r - lane, x, lane, v);
                });
            if (!ok) break;
        }
        if (FORM == kFormRows && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    if constexpr (FORM == kFormSplit) {
        // every CTA's partial tile is in its own shared memory: column c is added over the ranks, in rank
        // order, by the CTA c mod nrank
        cluster_sync();
        if (threadIdx.x < kMmEpiThreads && tile0 < tiles) {
            uint32_t tr, tc;
            tile_at(p, tile0, tr, tc);
            const uint32_t at_row = threadIdx.x & 127, r = tr * 128 + at_row;
            if (r < p.rows) {
                #pragma unroll 2
                for (uint32_t c = rank + (threadIdx.x >> 7) * nrank; c < (uint32_t)BN && tc * BN + c < p.cols; c += 2 * nrank) {
                    float v = 0.0f;
                    for (uint32_t q = 0; q < nrank; ++q) {
                        uint32_t at;
                        float x;
                        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem0 + (c * 128 + at_row) * 4), "r"(q));
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
                        v += x;
                    }
                    const uint64_t i = (uint64_t)(tc * BN + c) * p.ldo + r;
                    store_out<ODT>(p.out, i, p.accumulate ? v + load_out<ODT>(p.out, i) : v);
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
    if (stop && warp == 8 && leader)
        for (uint32_t b = issued > (uint32_t)S::kStages ? issued - S::kStages : 0; b < issued; ++b)
            mbar_drain(full(b % S::kStages), (b / S::kStages) & 1);
    if constexpr (CTAS == 2 || FORM == kFormSplit) cluster_sync();              // nothing of the other CTAs is in flight any more
    fence_after();
    if (threadIdx.x == 0 && stop && p.status != nullptr) *p.status = (uint32_t)LGN_ERR_TIMEOUT;
    if (warp == 9) {
        if constexpr (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" :: "r"(tmem));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem));
    }
}

// k = 0: nothing is added.
template <int ODT>
__global__ void __launch_bounds__(256) zero_rows_kernel(void *out, uint64_t ldo, uint32_t rows, uint32_t cols) {
    dep_wait();
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < (uint64_t)rows * cols; i += (uint64_t)gridDim.x * 256)
        store_out<ODT>(out, (i / cols) * ldo + i % cols, 0.0f);
}

// The kernels a call may take, with what a call of each costs on a B200, in microseconds: `start` once, `step` for 128 of k of
// a tile, `tile` for a tile beyond that (fitted to 60 products from 4 x 1024 x 1024 to 4096^3).  The fits leave errors of up to a
// fifth, about as much as neighbouring kernels differ; what they must get right is which side of
//   64 x k shares       few tokens: (4, 4096, 4096) 7.5 us in 4 shares, 10.2 whole, 9.8 with pairs of 128
//   pairs of 128        (512, 4096, 4096) 11.5 us, 13.3 with lone 128, 16.0 with pairs of 256
//   lone 128            where pairs would need a second round: (777, 2504, 1000) 7.0 us against 9.8
//   pairs of 256 / 192  (4096, 4096, 4096) 54 us in bf16, 57 with pairs of 128; 60 in fp32, 66 with pairs of 128
// a call lies on.
struct MmKernel { const void *fn; int bn, ctas, form, odt, smem, box; float start, step, tile; };
#define LGN_MM(BN, C, F, O, A, S, T) {reinterpret_cast<const void *>(&fp8_matmul_kernel<BN, C, F, O>), BN, C, F, O, MmShape<BN, C, O>::kSmem, MmShape<BN, C, O>::kBoxRows, A, S, T}
static const MmKernel kMmKernels[] = {
    LGN_MM(64, 1, kFormSwap, LGN_F32, 2.4f, 0.2f, 0.4f), LGN_MM(64, 1, kFormSplit, LGN_F32, 2.4f, 0.2f, 0.4f),
    LGN_MM(64, 1, kFormSwap, LGN_BF16, 2.4f, 0.2f, 0.1f), LGN_MM(64, 1, kFormSplit, LGN_BF16, 2.4f, 0.2f, 0.1f),
    LGN_MM(128, 1, kFormRows, LGN_F32, 3.0f, 0.25f, 1.0f), LGN_MM(128, 1, kFormSwap, LGN_F32, 3.0f, 0.25f, 1.3f),
    LGN_MM(128, 1, kFormRows, LGN_BF16, 3.0f, 0.24f, 0.4f), LGN_MM(128, 1, kFormSwap, LGN_BF16, 3.0f, 0.24f, 0.7f),
    LGN_MM(128, 2, kFormRows, LGN_F32, 3.2f, 0.18f, 1.3f), LGN_MM(128, 2, kFormSwap, LGN_F32, 3.2f, 0.18f, 1.6f),
    LGN_MM(128, 2, kFormRows, LGN_BF16, 3.2f, 0.17f, 0.9f), LGN_MM(128, 2, kFormSwap, LGN_BF16, 3.2f, 0.17f, 1.2f),
    LGN_MM(192, 2, kFormRows, LGN_F32, 3.3f, 0.22f, 2.2f), LGN_MM(192, 2, kFormSwap, LGN_F32, 3.3f, 0.22f, 2.5f),
    LGN_MM(256, 2, kFormRows, LGN_BF16, 3.3f, 0.3f, 1.1f), LGN_MM(256, 2, kFormSwap, LGN_BF16, 3.3f, 0.3f, 1.4f)};
#undef LGN_MM
constexpr int kMmCount = (int)(sizeof kMmKernels / sizeof kMmKernels[0]);

// rows x k codes, boxes of box_rows x 128 bytes; what lies outside reads as zero codes.
static bool make_map(CUtensorMap *m, const void *codes, uint64_t rows, uint64_t k, uint32_t box_rows) {
    const cuuint64_t dim[2] = {k, rows}, stride[1] = {fp8_pitch(k)};
    const cuuint32_t box[2] = {128, box_rows}, es[2] = {1, 1};
    return encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(codes), dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scale tiles as rows of 128 words.
static bool make_scale_map(CUtensorMap *m, const void *scales, uint64_t tiles) {
    const cuuint64_t dim[2] = {128, tiles}, stride[1] = {512};
    const cuuint32_t box[2] = {128, 1}, es[2] = {1, 1};
    return encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void *>(scales), dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The output: boxes of 32 rows x 128 bytes.  Needs rows aligned to, and a multiple of, 16 bytes.
static bool make_out_map(CUtensorMap *m, void *out, uint64_t rows, uint64_t cols, uint64_t ldo, int odt) {
    const uint64_t es = odt == LGN_F32 ? 4 : 2;
    const cuuint64_t dim[2] = {cols, rows}, stride[1] = {ldo * es};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32}, st[2] = {1, 1};
    return encode_tiled()(m, odt == LGN_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, out, dim, stride, box, st,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The kernels need more dynamic shared memory than the default limit; raised once per device and kernel.
static bool allow_smem(int kernel) {
    static std::mutex guard;
    static bool done[64][kMmCount];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
    std::lock_guard<std::mutex> lock(guard);
    if (dev < 64 && done[dev][kernel]) return true;
    if (cudaFuncSetAttribute(kMmKernels[kernel].fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmKernels[kernel].smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    if (dev < 64) done[dev][kernel] = true;
    return true;
}

// Clusters of 2, 4 or 8 CTAs of a kernel that the device can run at once (found once per device and kernel).
static int active_clusters(int kernel, int size_log2) {
    static std::mutex guard;
    static int found[64][kMmCount][4];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || !allow_smem(kernel)) return 0;
    std::lock_guard<std::mutex> lock(guard);
    int &n = found[dev][kernel][size_log2];
    if (n == 0) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1u << size_log2;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.gridDim = dim3(1u << size_log2);
        cfg.blockDim = dim3(kMmThreads);
        cfg.dynamicSmemBytes = (size_t)kMmKernels[kernel].smem;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int c = 0;
        if (cudaOccupancyMaxActiveClusters(&c, kMmKernels[kernel].fn, &cfg) != cudaSuccess) { (void)cudaGetLastError(); c = 0; }
        n = c > 0 ? c : -1;
    }
    return n > 0 ? n : 0;
}

struct MmPlan { int kernel; uint32_t split, split_groups; };

// The kernel of least estimated time: rounds of the grid times the cost of a tile.
static MmPlan plan_matmul(uint64_t m, uint64_t n, uint64_t kblocks, bool vec, int odt, int sms) {
    MmPlan best = {-1, 1, 0};
    const uint64_t groups = (kblocks + 3) / 4;
    double best_cost = 1e300;
    for (int i = 0; i < kMmCount; ++i) {
        const MmKernel &q = kMmKernels[i];
        if (q.odt != odt || (q.form == kFormRows && !vec)) continue;
        const uint64_t rows = 128 * (uint64_t)q.ctas, bn = (uint64_t)q.bn, r = q.form == kFormRows ? m : n, c = q.form == kFormRows ? n : m;
        const uint64_t tiles = ((r + rows - 1) / rows) * ((c + bn - 1) / bn), slots = (uint64_t)(sms / q.ctas);
        if (q.form != kFormSplit) {
            const double cost = q.start + (double)((tiles + slots - 1) / slots) * ((double)kblocks * q.step + q.tile);
            if (cost < best_cost) { best_cost = cost; best = {i, 1, 0}; }
            continue;
        }
        for (int l = 1; l <= 3; ++l) {
            // shares of whole groups of four blocks; a CTA adds up its part of min(c, bn) columns of each share
            const uint64_t per = (groups + (1u << l) - 1) >> l, s = (groups + per - 1) / per;
            if (s < 2 || tiles > (uint64_t)active_clusters(i, s > 4 ? 3 : s > 2 ? 2 : 1)) continue;
            const double cost = (double)(per * 4 < kblocks ? per * 4 : kblocks) * q.step + q.start + q.tile + 0.5 + 0.05 * (double)(c < bn ? c : bn);
            if (cost < best_cost) { best_cost = cost; best = {i, (uint32_t)s, (uint32_t)per}; }
        }
    }
    return best;
}

}  // namespace lgn

using namespace lgn;

static lgn_status matmul(const void *a, const void *a_scales, lgn_fp8 a_fmt, const void *b, const void *b_scales, lgn_fp8 b_fmt,
                         uint64_t m, uint64_t n, uint64_t k, void *out, uint64_t ldo, lgn_dtype out_dt, int accumulate,
                         uint32_t *status_dev, void *stream, bool withhold) {
    if ((a_fmt != LGN_E4M3 && a_fmt != LGN_E5M2) || (b_fmt != LGN_E4M3 && b_fmt != LGN_E5M2)) return LGN_ERR_INVALID_ARG;
    if (out_dt != LGN_F32 && out_dt != LGN_BF16) return LGN_ERR_INVALID_ARG;
    if (m > kFp8MaxDim || n > kFp8MaxDim || k > kFp8MaxDim) return LGN_ERR_UNSUPPORTED;
    if (m == 0 || n == 0) return LGN_OK;
    if (ldo < n || ldo > (1ull << 40)) return LGN_ERR_INVALID_ARG;
    const uint64_t es = out_dt == LGN_F32 ? 4 : 2, ob = matrix_bytes(m, n, ldo, es);
    if (ob == 0 || out == nullptr || !aligned_to(out, es) || !aligned_to(status_dev, 4)) return LGN_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (k == 0) {
        if (accumulate) return LGN_OK;
        uint32_t rows = (uint32_t)m, cols = (uint32_t)n;
        void *args[] = {&out, &ldo, &rows, &cols};
        const void *fn = out_dt == LGN_F32 ? reinterpret_cast<const void *>(&zero_rows_kernel<LGN_F32>) : reinterpret_cast<const void *>(&zero_rows_kernel<LGN_BF16>);
        const uint64_t want = (m * n + 255) / 256;
        return launch_dependent(fn, dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), args, 0, stream);
    }
    if (a == nullptr || b == nullptr || a_scales == nullptr || b_scales == nullptr) return LGN_ERR_INVALID_ARG;
    if (!aligned_to(a, 16) || !aligned_to(b, 16) || !aligned_to(a_scales, 16) || !aligned_to(b_scales, 16)) return LGN_ERR_INVALID_ARG;
    if (ranges_overlap(out, ob, a, lgn_fp8_codes_bytes(m, k)) || ranges_overlap(out, ob, b, lgn_fp8_codes_bytes(n, k)) ||
        ranges_overlap(out, ob, a_scales, lgn_fp8_scales_bytes(m, k)) || ranges_overlap(out, ob, b_scales, lgn_fp8_scales_bytes(n, k)))
        return LGN_ERR_INVALID_ARG;
    if (sms < 1 || encode_tiled() == nullptr) return LGN_ERR_CUDA;
    // TMA stores: aligned rows, and whole 16-byte pieces (a row's last piece is written whole, beyond the n-th element too)
    const bool vec = aligned_to(out, 16) && (ldo * es) % 16 == 0 && (n * es) % 16 == 0;
    const uint64_t kblocks = (k + 127) / 128;
    const MmPlan plan = plan_matmul(m, n, kblocks, vec, out_dt, sms);
    if (plan.kernel < 0) return LGN_ERR_UNSUPPORTED;
    const MmKernel &q = kMmKernels[plan.kernel];
    const bool swap = q.form != kFormRows;
    const uint32_t bn = (uint32_t)q.bn, tile_rows = 128 * (uint32_t)q.ctas;
    MmArgs p = {};
    const void *cr = swap ? b : a, *cc = swap ? a : b;
    p.rows = (uint32_t)(swap ? n : m);
    p.cols = (uint32_t)(swap ? m : n);
    p.fmt_rows = (uint32_t)(swap ? b_fmt : a_fmt);
    p.fmt_cols = (uint32_t)(swap ? a_fmt : b_fmt);
    p.out = out; p.ldo = ldo; p.status = status_dev;
    p.kblocks = (uint32_t)kblocks;
    p.groups = (uint32_t)((kblocks + 3) / 4);
    p.tiles_r = (p.rows + tile_rows - 1) / tile_rows;
    p.tiles_c = (p.cols + bn - 1) / bn;
    p.split_groups = plan.split_groups;
    p.accumulate = accumulate != 0;
    p.withhold = withhold;
    const uint64_t tiles = (uint64_t)p.tiles_r * p.tiles_c, slots = (uint64_t)(sms / q.ctas);
    if (tiles > 0x3fffffffull || (uint64_t)((p.rows + 127) / 128) * p.groups > 0x7fffffffull || (uint64_t)((p.cols + 127) / 128) * p.groups > 0x7fffffffull)
        return LGN_ERR_UNSUPPORTED;                                             // TMA coordinates are 32-bit
    CUtensorMap mr, mc, sr, sc, mo = {};
    if (q.form == kFormRows && !make_out_map(&mo, out, m, n, ldo, out_dt)) return LGN_ERR_CUDA;
    if (!make_map(&mr, cr, p.rows, k, 128) || !make_map(&mc, cc, p.cols, k, (uint32_t)q.box)) return LGN_ERR_CUDA;
    if (!make_scale_map(&sr, swap ? b_scales : a_scales, (uint64_t)((p.rows + 127) / 128) * p.groups) ||
        !make_scale_map(&sc, swap ? a_scales : b_scales, (uint64_t)((p.cols + 127) / 128) * p.groups)) return LGN_ERR_CUDA;
    if (!allow_smem(plan.kernel)) return LGN_ERR_CUDA;
    const uint64_t grid = q.form == kFormSplit ? tiles * plan.split : (tiles < slots ? tiles : slots);
    log_line("fp8_matmul: m %llu n %llu k %llu, %s, tile %u x %u, form %d, split %u, %llu tiles", (unsigned long long)m, (unsigned long long)n,
             (unsigned long long)k, q.ctas == 2 ? "pairs" : "single", tile_rows, bn, q.form, plan.split, (unsigned long long)tiles);
    void *args[] = {&mr, &mc, &sr, &sc, &mo, &p};
    return launch_dependent(q.fn, dim3((unsigned)grid * (unsigned)q.ctas), dim3(kMmThreads), args, (size_t)q.smem, stream,
                            q.form == kFormSplit ? plan.split : (unsigned)q.ctas);
}

extern "C" lgn_status lgn_fp8_matmul(const void *a, const void *a_scales, lgn_fp8 a_fmt, const void *b, const void *b_scales, lgn_fp8 b_fmt,
                                     uint64_t m, uint64_t n, uint64_t k, void *out, uint64_t ldo, lgn_dtype out_dt, int accumulate,
                                     uint32_t *status_dev, void *stream) {
    return matmul(a, a_scales, a_fmt, b, b_scales, b_fmt, m, n, k, out, ldo, out_dt, accumulate, status_dev, stream, false);
}

extern "C" lgn_status lgn_selftest_matmul_wait_expires(const void *a, const void *a_scales, const void *b, const void *b_scales,
                                                       uint64_t m, uint64_t n, uint64_t k, void *out, lgn_dtype out_dt,
                                                       uint32_t *status_dev, void *stream) {
    if (status_dev == nullptr || k == 0) return LGN_ERR_INVALID_ARG;
    return matmul(a, a_scales, LGN_E4M3, b, b_scales, LGN_E4M3, m, n, k, out, n, out_dt, 0, status_dev, stream, true);
}
