// Host side of the grouped products: checks, the choice of a kernel, tensor maps, launches.
#include <mutex>

#include "lgn_fp8.cuh"
#include "lgn_grouped.cuh"
#include "lgn_log.h"

namespace lgn {

constexpr uint64_t kGmMaxDim = 1ull << 30, kGmMaxGroups = 1ull << 20;
constexpr uint64_t kGmMaxInt8K = 1ull << 17;             // 127 * 127 * 2^17 < 2^31: the integer sum cannot overflow

// The kernels need more dynamic shared memory than the default limit; raised once per device and kernel.
static bool gm_allow_smem(int list, int i, const GmKernel &q) {
    static std::mutex guard;
    static bool done[64][4][16];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
    std::lock_guard<std::mutex> lock(guard);
    if (dev < 64 && i < 16 && done[dev][list][i]) return true;
    if (cudaFuncSetAttribute(q.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, q.smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    if (dev < 64 && i < 16) done[dev][list][i] = true;
    return true;
}

// x (contiguous) by y by z elements, boxes of 128 bytes by `box_y`; what lies outside reads as zero and is not written.
static bool gm_map(CUtensorMap *m, CUtensorMapDataType type, uint64_t es, const void *at, uint64_t x, uint64_t y, uint64_t z, uint64_t pitch, uint64_t group, uint32_t box_y) {
    const cuuint64_t dim[3] = {x, y, z}, stride[2] = {pitch * es, z > 1 ? group * es : pitch * es};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / es), box_y, 1}, step[3] = {1, 1, 1};
    return encode_tiled()(m, type, 3, const_cast<void *>(at), dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

enum GmProduct { kGmForward = 0, kGmInput = 1, kGmWeight = 2, kGmIntegers = 3 };

struct GmOperand { const void *at; uint64_t x, y, z, pitch, group; };     // as in memory: x contiguous, y rows, z matrices

struct GmPlan { int kernel; uint32_t split, split_steps; uint64_t row_tiles; };

// The height (of the groups' rows, or of the gradient's matrices) and the width of a kernel's tile.
static uint64_t gm_height(const GmKernel &q) { return q.form == kGmSwap || q.form == kGmTurn ? (uint64_t)q.bn : 128 * (uint64_t)q.ctas; }
static uint64_t gm_width(const GmKernel &q) { return q.form == kGmSwap || q.form == kGmTurn ? 128 * (uint64_t)q.ctas : (uint64_t)q.bn; }

// Row tiles of `height` of all groups: an upper bound, and what is likely.
static uint64_t gm_most_tiles(uint64_t rows, uint64_t groups, uint64_t height) {
    return groups == 1 ? (rows + height - 1) / height : rows / height + (groups < rows ? groups : rows);
}
static double gm_likely_tiles(uint64_t rows, uint64_t groups, uint64_t height) {
    if (groups == 1 || rows == 0) return (double)((rows + height - 1) / height);
    const double met = (double)(groups < rows ? groups : rows), each = (double)rows / met / (double)height + 0.5;
    return met * (each < 1.0 ? 1.0 : each);
}

// What the kernels cost on a B200, in microseconds: `start` once, `step` for 128 bytes of the contraction of a tile (and `full` times the share of its
// columns that are in use), `tile` for a tile beyond that (bf16 and fp32 outputs); the memory's part is 6.9 TB/s.  Fitted to 213 products, half of them drawn: 1 to
// 32768 rows, 1 to 128 groups whose sizes spread by a factor of 8, widths from 96 to 8192.  The estimates are off by 17 % in the mean, what they choose
// is 2 % slower than the fastest.  Which side of these a call lies on is what they must get right:
//   swapped, 4 shares    2 rows, 8 x 4096 x 4096: 12.8 us, turned pairs 15.6, pairs 24
//   swapped, turned      64 rows, the same: 45 us, 46; pairs 52, lone 128 48
//   turned pairs         2048 rows, the same: 70 us, pairs 81, lone 128 93; 5003 rows, 60 x 1448 x 1000 in fp32: 38, 50, 52
//   pairs                32768 rows, 8 x 1024 x 1024: 56 us, turned 58.5, lone 128 70
//   lone 128             300 rows, 4 x 512 x 512: 5.5 us, turned 6.5, pairs 7.4
//   pairs of 128         8-bit integers, 512 rows, 4096 x 4096: 10.9 us, lone 128 11.7, pairs 15.9, turned 18.2
//   rows shared out      gradient of 2 x 512 x 512 over 32768 rows: 35 us in 4 shares, 113 with lone 128, 134 with pairs
struct GmCost { int form, bn, ctas; float start, step, full, tile[2]; };     // tile: by LGN_F32, LGN_BF16
static const GmCost kGmCosts[] = {
    {kGmRows, 256, 2, 2.3f, 0.30f, 0.0f, {2.7f, 1.4f}}, {kGmTurn, 256, 2, 2.5f, 0.11f, 0.20f, {2.7f, 2.0f}}, {kGmRows, 128, 2, 3.1f, 0.16f, 0.0f, {2.1f, 1.1f}},
    {kGmRows, 128, 1, 2.6f, 0.27f, 0.0f, {2.4f, 1.1f}}, {kGmSwap, 32, 1, 1.2f, 0.23f, 0.0f, {4.6f, 3.8f}},  {kGmSwap, 64, 1, 1.2f, 0.23f, 0.0f, {5.1f, 5.4f}},
    {kGmGrad, 256, 2, 5.1f, 0.45f, 0.0f, {2.4f, 1.4f}}, {kGmGrad, 128, 1, 4.1f, 0.42f, 0.0f, {1.0f, 0.6f}}, {kGmShare, 128, 1, 5.2f, 0.45f, 0.0f, {4.0f, 2.1f}}};
static_assert(LGN_F32 == 0 && LGN_BF16 == 1, "GmCost::tile");

// The kernel of least estimated time: rounds of the grid times the cost of a tile, or the memory's time where that is longer.  What the sizes of the groups
// are is known on the device alone; equal ones are assumed here.  `bytes`: what the product reads and writes.  `vec`: the output's rows are whole 16-byte
// pieces; where they are not, lanes that store along a row take 4 bytes each, and tiles cost half as much again (5994 rows over 42 experts,
// 336 -> 2355: pairs 37 us, 27 for 2360; turned tiles 24 and 22).
static GmPlan gm_plan(const GmKernels &list, uint64_t rows, uint64_t groups, uint64_t m, uint64_t n, uint64_t steps, double bytes, bool vec, int odt, int sms) {
    GmPlan best = {-1, 1, 0, 0};
    double best_cost = 1e300;
    for (int i = 0; i < list.count; ++i) {
        const GmKernel &q = list.first[i];
        const GmCost *c = nullptr;
        for (const GmCost &k : kGmCosts) if (k.form == q.form && k.bn == q.bn && k.ctas == q.ctas) c = &k;
        if (q.odt != odt || c == nullptr) continue;
        const bool grad = q.form == kGmGrad || q.form == kGmShare, one = q.form == kGmSwap || q.form == kGmShare;
        const uint64_t height = gm_height(q), cols = (n + gm_width(q) - 1) / gm_width(q), fixed = groups * ((m + height - 1) / height);
        const double row_tiles = grad ? (double)fixed : gm_likely_tiles(rows, groups, height), tiles = row_tiles * (double)cols;
        const uint64_t most = grad ? fixed : gm_most_tiles(rows, groups, height);
        const double all_steps = grad ? (double)rows / (double)groups / 64.0 + 0.5 : (double)steps, slots = (double)(q.form == kGmSwap ? 2 * sms : sms / q.ctas);
        const double used = row_tiles > 0.0 ? (double)rows / row_tiles / (double)height : 1.0, step = c->step + c->full * (used < 1.0 ? used : 1.0);
        for (uint32_t split = q.form == kGmShare ? 2 : 1; split <= (one ? 8u : 1u); split *= 2) {
            if (split > 1 && ((double)split > all_steps || tiles * split > 2.0 * slots)) break;
            const double share = split > 1 ? (double)(uint64_t)((all_steps + split - 1) / split) : all_steps;
            double rounds = tiles * split / slots;
            rounds = rounds < 1.0 ? 1.0 : rounds < 4.0 ? (double)(uint64_t)(rounds + 0.999) : rounds + 0.5;
            const bool slow = !vec && (q.form == kGmRows || q.form == kGmGrad);
            const double work = rounds * (share * step + c->tile[odt]) * (slow ? 1.5 : 1.0) + (split > 1 ? 0.58 + 0.07 * split : 0.0), memory = bytes / 6.9e6;
            const double cost = c->start + (work > memory ? work : memory) + 0.04 * work;
            if (cost < best_cost) {
                best_cost = cost;
                best = {i, split, (uint32_t)((steps + split - 1) / split), most};
            }
        }
    }
    return best;
}

// One of the products; `a`: the activations (gradient: dY), `b`: the weights (gradient: X).
static lgn_status gm_run(GmProduct which, const GmOperand &a, const GmOperand &b, GmArgs &p, uint64_t k, int odt, void *stream) {
    const GmKernels list = which == kGmForward ? gm_forward_kernels() : which == kGmInput ? gm_input_kernels() : which == kGmWeight ? gm_weight_kernels() : gm_int8_kernels();
    const bool int8 = which == kGmIntegers, grad = which == kGmWeight;
    const uint64_t keep = int8 ? 128 : 64, steps = grad ? 0 : (k + keep - 1) / keep;
    const int sms = sm_count();
    if (sms < 1 || encode_tiled() == nullptr) return LGN_ERR_CUDA;
    const uint64_t es = odt == LGN_F32 ? 4 : 2, ies = int8 ? 1 : 2;
    const double met = (double)(p.groups < p.rows ? p.groups : p.rows);
    const double bytes = grad ? (double)ies * p.rows * ((double)p.m + p.n) + (double)es * p.groups * p.m * p.n
                              : (double)ies * (double)k * (p.rows + met * p.n) + (double)es * p.rows * p.n;
    p.vec = aligned_to(p.out, 16) && (p.ldo * es) % 16 == 0 && (p.n * es) % 16 == 0 && (!grad || p.groups == 1 || (p.out_group * es) % 16 == 0);
    const GmPlan plan = gm_plan(list, p.rows, p.groups, p.m, p.n, steps, bytes, p.vec != 0, odt, sms);
    if (plan.kernel < 0) return LGN_ERR_UNSUPPORTED;
    const GmKernel &q = list.first[plan.kernel];
    const uint64_t height = gm_height(q), width = gm_width(q);
    const bool turned = q.form == kGmSwap || q.form == kGmTurn;
    p.steps = (uint32_t)steps;
    p.split_steps = plan.split_steps;
    p.tiles_c = (uint32_t)((p.n + width - 1) / width);
    p.tiles_r = grad ? (uint32_t)((p.m + height - 1) / height) : 0;
    const uint64_t most = plan.row_tiles * p.tiles_c;
    if (most > 0x3fffffffull || most * plan.split > 0x7fffffffull) return LGN_ERR_UNSUPPORTED;

    CUtensorMap ma = {}, mb = {};
    const CUtensorMapDataType type = int8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const bool any = p.rows > 0 && (grad || steps > 0);                   // anything to copy in
    // the MMA's rows come from the activations, or, swapped, from the weights
    const GmOperand &r = turned ? b : a, &c = turned ? a : b;
    const bool one = q.form == kGmSwap || q.form == kGmShare;
    const bool boxes_r = grad || (turned && !q.along), boxes_c = grad || (q.form == kGmRows && !q.along);
    if (any && (!gm_map(&ma, type, ies, r.at, r.x, r.y, r.z, r.pitch, r.group, boxes_r ? 64 : 128) ||
                !gm_map(&mb, type, ies, c.at, c.x, c.y, c.z, c.pitch, c.group, boxes_c ? 64 : q.form == kGmTurn ? 32 : (uint32_t)(q.bn / q.ctas)))) return LGN_ERR_CUDA;
    if (!gm_allow_smem(which, plan.kernel, q)) return LGN_ERR_CUDA;
    const uint64_t slots = (uint64_t)(sms / q.ctas);
    uint64_t grid = one ? most * plan.split : (most < slots ? most : slots) * (uint64_t)q.ctas;
    if (grid == 0) grid = (uint64_t)q.ctas * plan.split;
    log_line("grouped: %s, rows %u groups %u m %u n %u, %llu steps, tile %llu x %llu, form %d, split %u, up to %llu tiles",
             which == kGmForward ? "X W^T" : which == kGmInput ? "X W" : which == kGmWeight ? "dY^T X" : "8-bit X W^T", p.rows, p.groups, p.m, p.n, (unsigned long long)steps,
             (unsigned long long)height, (unsigned long long)width, q.form, plan.split, (unsigned long long)most);
    void *args[] = {&ma, &mb, &p};
    return launch_dependent(q.fn, dim3((unsigned)grid), dim3((unsigned)gm_threads(q.form)), args, (size_t)q.smem, stream, one ? plan.split : (unsigned)q.ctas);
}

// Checks that the entries share: group offsets and the output.
static lgn_status gm_check(const void *offsets, int offset_bits, uint64_t groups, uint64_t rows, uint64_t n, lgn_dtype out_dt, const uint32_t *status_dev) {
    if (out_dt != LGN_F32 && out_dt != LGN_BF16) return LGN_ERR_INVALID_ARG;
    if (offset_bits != 32 && offset_bits != 64) return LGN_ERR_INVALID_ARG;
    if (groups == 0 || !aligned_to(offsets, (uintptr_t)offset_bits / 8) || !aligned_to(status_dev, 4)) return LGN_ERR_INVALID_ARG;
    if (rows > kGmMaxDim || n > kGmMaxDim || groups > kGmMaxGroups) return LGN_ERR_UNSUPPORTED;
    return LGN_OK;
}

// A bf16 operand that TMA can read: rows and matrices whole 16-byte pieces apart.
static bool gm_readable(const GmOperand &o) {
    return o.at != nullptr && aligned_to(o.at, 16) && o.pitch >= o.x && o.pitch % 8 == 0 && o.pitch <= (1ull << 38) &&
           (o.z <= 1 || (o.group % 8 == 0 && o.group <= (1ull << 38)));
}
// Bytes from an operand's first to its last element; 0: more than memory can have, or matrices that overlap.
static uint64_t gm_bytes(const GmOperand &o, uint64_t es) {
    const uint64_t one = matrix_bytes(o.y, o.x, o.pitch, es);
    if (o.z <= 1 || one == 0) return one;
    if (o.group < one / es || (o.z - 1) > ((1ull << 61) / es) / o.group) return 0;
    return (o.z - 1) * o.group * es + one;
}

}  // namespace lgn

using namespace lgn;

static lgn_status grouped_matmul(const void *x, uint64_t ldx, const void *w, uint64_t ldw, uint64_t w_group, int transposed,
                                 const void *offsets, int offset_bits, uint64_t groups, uint64_t rows, uint64_t n, uint64_t k,
                                 void *out, uint64_t ldo, lgn_dtype out_dt, int zero_rest, uint32_t *status_dev, void *stream, bool withhold) {
    const lgn_status bad = gm_check(offsets, offset_bits, groups, rows, n, out_dt, status_dev);
    if (bad != LGN_OK) return bad;
    if (k > kGmMaxDim) return LGN_ERR_UNSUPPORTED;
    if (rows == 0 || n == 0) return LGN_OK;
    const uint64_t es = out_dt == LGN_F32 ? 4 : 2;
    if (offsets == nullptr || out == nullptr || !aligned_to(out, es) || ldo < n || ldo > (1ull << 38)) return LGN_ERR_INVALID_ARG;
    const uint64_t ob = matrix_bytes(rows, n, ldo, es);
    const GmOperand a = {x, k, rows, 1, ldx, 0}, b = {w, transposed ? n : k, transposed ? k : n, groups, ldw, w_group};
    if (ob == 0 || ranges_overlap(out, ob, offsets, (groups + 1) * (uint64_t)offset_bits / 8)) return LGN_ERR_INVALID_ARG;
    if (k > 0) {
        if (!gm_readable(a) || !gm_readable(b)) return LGN_ERR_INVALID_ARG;
        const uint64_t ab = gm_bytes(a, 2), bb = gm_bytes(b, 2);
        if (ab == 0 || bb == 0 || ranges_overlap(out, ob, x, ab) || ranges_overlap(out, ob, w, bb)) return LGN_ERR_INVALID_ARG;
    }
    GmArgs p = {};
    p.out = static_cast<char *>(out); p.ldo = ldo; p.offsets = offsets; p.offsets64 = offset_bits == 64; p.status = status_dev;
    p.rows = (uint32_t)rows; p.groups = (uint32_t)groups; p.n = (uint32_t)n; p.zero_rest = zero_rest != 0; p.withhold = withhold;
    return gm_run(transposed ? kGmInput : kGmForward, a, b, p, k, out_dt, stream);
}

static lgn_status weight_grad(const void *dy, uint64_t lddy, const void *x, uint64_t ldx, const void *offsets, int offset_bits,
                              uint64_t groups, uint64_t rows, uint64_t m, uint64_t n, void *out, uint64_t ldo, uint64_t out_group,
                              lgn_dtype out_dt, int accumulate, uint32_t *status_dev, void *stream, bool withhold) {
    const lgn_status bad = gm_check(offsets, offset_bits, groups, rows, n, out_dt, status_dev);
    if (bad != LGN_OK) return bad;
    if (m > kGmMaxDim) return LGN_ERR_UNSUPPORTED;
    if (m == 0 || n == 0) return LGN_OK;
    const uint64_t es = out_dt == LGN_F32 ? 4 : 2;
    if (offsets == nullptr || out == nullptr || !aligned_to(out, es) || ldo < n || ldo > (1ull << 38) || (groups > 1 && out_group > (1ull << 38))) return LGN_ERR_INVALID_ARG;
    const GmOperand a = {dy, m, rows, 1, lddy, 0}, b = {x, n, rows, 1, ldx, 0}, o = {out, n, m, groups, ldo, out_group};
    const uint64_t ob = gm_bytes(o, es);
    if (ob == 0 || ranges_overlap(out, ob, offsets, (groups + 1) * (uint64_t)offset_bits / 8)) return LGN_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!gm_readable(a) || !gm_readable(b)) return LGN_ERR_INVALID_ARG;
        const uint64_t ab = gm_bytes(a, 2), bb = gm_bytes(b, 2);
        if (ab == 0 || bb == 0 || ranges_overlap(out, ob, dy, ab) || ranges_overlap(out, ob, x, bb)) return LGN_ERR_INVALID_ARG;
    }
    GmArgs p = {};
    p.out = static_cast<char *>(out); p.ldo = ldo; p.out_group = out_group; p.offsets = offsets; p.offsets64 = offset_bits == 64; p.status = status_dev;
    p.rows = (uint32_t)rows; p.groups = (uint32_t)groups; p.m = (uint32_t)m; p.n = (uint32_t)n; p.accumulate = accumulate != 0; p.withhold = withhold;
    return gm_run(kGmWeight, a, b, p, 0, out_dt, stream);
}

static lgn_status int8_matmul(const void *a, const float *a_scales, const void *b, const float *b_scales,
                              const void *offsets, int offset_bits, uint64_t groups, uint64_t m, uint64_t n, uint64_t k,
                              void *out, uint64_t ldo, lgn_dtype out_dt, int zero_rest, uint32_t *status_dev, void *stream, bool withhold) {
    const lgn_status bad = gm_check(offsets, offset_bits, groups, m, n, out_dt, status_dev);
    if (bad != LGN_OK) return bad;
    if (k > kGmMaxInt8K || groups * n > kGmMaxDim) return LGN_ERR_UNSUPPORTED;
    if (m == 0 || n == 0) return LGN_OK;
    const uint64_t es = out_dt == LGN_F32 ? 4 : 2, pitch = fp8_pitch(k);
    if ((offsets == nullptr && groups != 1) || out == nullptr || !aligned_to(out, es) || ldo < n || ldo > (1ull << 38)) return LGN_ERR_INVALID_ARG;
    const uint64_t ob = matrix_bytes(m, n, ldo, es);
    if (ob == 0 || ranges_overlap(out, ob, offsets, offsets != nullptr ? (groups + 1) * (uint64_t)offset_bits / 8 : 0)) return LGN_ERR_INVALID_ARG;
    if (k > 0) {
        if (a == nullptr || b == nullptr || a_scales == nullptr || b_scales == nullptr) return LGN_ERR_INVALID_ARG;
        if (!aligned_to(a, 16) || !aligned_to(b, 16) || !aligned_to(a_scales, 4) || !aligned_to(b_scales, 4)) return LGN_ERR_INVALID_ARG;
        if (ranges_overlap(out, ob, a, m * pitch) || ranges_overlap(out, ob, b, groups * n * pitch) ||
            ranges_overlap(out, ob, a_scales, 4 * m) || ranges_overlap(out, ob, b_scales, 4 * groups * n)) return LGN_ERR_INVALID_ARG;
    }
    const GmOperand x = {a, k, m, 1, pitch, 0}, w = {b, k, n, groups, pitch, n * pitch};
    GmArgs p = {};
    p.out = static_cast<char *>(out); p.ldo = ldo; p.offsets = offsets; p.offsets64 = offset_bits == 64; p.status = status_dev;
    p.rows = (uint32_t)m; p.groups = (uint32_t)groups; p.n = (uint32_t)n; p.zero_rest = zero_rest != 0; p.withhold = withhold;
    // Over nothing the scales may be absent or without a meaning, and the integer kernels read them: the bf16 ones write the same zeros.
    if (k == 0) return gm_run(kGmForward, x, w, p, 0, out_dt, stream);
    p.row_scales = a_scales; p.col_scales = b_scales;
    return gm_run(kGmIntegers, x, w, p, k, out_dt, stream);
}

extern "C" lgn_status lgn_grouped_matmul(const void *x, uint64_t ldx, const void *w, uint64_t ldw, uint64_t w_group, int transposed,
                                         const void *offsets, int offset_bits, uint64_t groups, uint64_t rows, uint64_t n, uint64_t k,
                                         void *out, uint64_t ldo, lgn_dtype out_dt, int zero_rest, uint32_t *status_dev, void *stream) {
    return grouped_matmul(x, ldx, w, ldw, w_group, transposed, offsets, offset_bits, groups, rows, n, k, out, ldo, out_dt, zero_rest, status_dev, stream, false);
}

extern "C" lgn_status lgn_grouped_weight_grad(const void *dy, uint64_t lddy, const void *x, uint64_t ldx, const void *offsets, int offset_bits,
                                              uint64_t groups, uint64_t rows, uint64_t m, uint64_t n, void *out, uint64_t ldo, uint64_t out_group,
                                              lgn_dtype out_dt, int accumulate, uint32_t *status_dev, void *stream) {
    return weight_grad(dy, lddy, x, ldx, offsets, offset_bits, groups, rows, m, n, out, ldo, out_group, out_dt, accumulate, status_dev, stream, false);
}

extern "C" lgn_status lgn_selftest_grouped_wait_expires(const void *a, const void *b, int gradient, const void *offsets, int offset_bits,
                                                        uint64_t groups, uint64_t rows, uint64_t n, uint64_t k, void *out, lgn_dtype out_dt,
                                                        uint32_t *status_dev, void *stream) {
    if (status_dev == nullptr || rows == 0 || k == 0) return LGN_ERR_INVALID_ARG;
    // The codes are at least as long as the scales: any floats do, nothing comes of them.
    if (gradient == 2) return int8_matmul(a, static_cast<const float *>(a), b, static_cast<const float *>(b), offsets, offset_bits, groups, rows, n, k, out, n, out_dt, 0,
                                          status_dev, stream, true);
    return gradient ? weight_grad(a, n, b, k, offsets, offset_bits, groups, rows, n, k, out, k, n * k, out_dt, 0, status_dev, stream, true)
                    : grouped_matmul(a, k, b, k, n * k, 0, offsets, offset_bits, groups, rows, n, k, out, n, out_dt, 0, status_dev, stream, true);
}

extern "C" lgn_status lgn_int8_matmul(const void *a, const float *a_scales, const void *b, const float *b_scales,
                                      const void *offsets, int offset_bits, uint64_t groups, uint64_t m, uint64_t n, uint64_t k,
                                      void *out, uint64_t ldo, lgn_dtype out_dt, int zero_rest, uint32_t *status_dev, void *stream) {
    return int8_matmul(a, a_scales, b, b_scales, offsets, offset_bits, groups, m, n, k, out, ldo, out_dt, zero_rest, status_dev, stream, false);
}
