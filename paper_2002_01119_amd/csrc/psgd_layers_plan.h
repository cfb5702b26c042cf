// Which kernel, tile and number of parts a call of the layers and losses takes: plain host arithmetic on sizes, types and the number of compute
// units, kept apart from the kernels so that a CPU build can say what a size runs.
#ifndef PSGD_LAYERS_PLAN_H
#define PSGD_LAYERS_PLAN_H

#include <cmath>
#include <cstddef>
#include <cstdint>
#include <initializer_list>
#include <iterator>

#include "psgd_layers.h"

namespace psgd {

constexpr int kWave = 64;

inline size_t up256(size_t b) { return (b + 255) / 256 * 256; }
inline int64_t parts_of(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of a launch along x: its work items are counted in 32 bits, and what is beyond is not started, without an error.  Larger calls are launched in
// slices of so many.
constexpr int64_t kMostGroups = 1 << 21;
template <typename F> void in_slices(int64_t groups, const F& launch) {      // launch(first, count)
    for (int64_t first = 0; first < groups; first += kMostGroups) launch(first, (unsigned)(groups - first < kMostGroups ? groups - first : kMostGroups));
}

// ------------------------------------------------------------------------------------------------ linear layer
constexpr int kRowBytes = 128;                     // a row of the LDS tile: 64 bf16 or 32 floats of k, as eight chunks of 16 bytes

struct Plan {
    int rows, cols, split;       // of a workgroup's tile; parts of k
    size_t bytes(int learners, int64_t m, int64_t n) const {
        return split > 1 ? up256((size_t)split * learners * m * n * sizeof(float)) : 0;
    }
};

// What a tile costs, in us: a step of 128 bytes of k with nothing else on the compute unit, the same when the unit is full (a share of it), and what
// comes before and after the steps.  Measured (products of 16 to 8192 a side, each tile with 1 to 32 parts of k; over 102 of them the choice costs 1 %
// more than the best tile would): large tiles do the most with what they read, small ones fill the chip and wait less, and tiles of 32 multiply few
// rows beyond the operand's (float, 7 x 4096 x 1512 -> 25: 40 us, by 64 x 64 68).  bf16 has none of those: its narrow products wait for memory.
struct TileCost {
    int rows, cols, resident;
    float alone, shared, ends;
};
constexpr TileCost kCostsBf16[] = {{256, 256, 1, 1.75f, 1.75f, 9.0f}, {128, 128, 2, 0.7f, 0.45f, 5.0f}, {64, 64, 4, 0.53f, 0.25f, 2.2f}};
constexpr TileCost kCostsFloat[] = {{256, 256, 1, 8.0f, 8.0f, 10.0f}, {128, 128, 2, 2.4f, 2.4f, 6.0f}, {64, 64, 4, 0.7f, 0.55f, 2.5f},
                                    {128, 32, 4, 0.7f, 0.55f, 2.5f}, {32, 128, 4, 0.7f, 0.55f, 2.5f}};

// One whole tile of k at most: there is no second one beside it in LDS, and one workgroup more fits a compute unit, where its registers do: not of the
// largest, nor of 128 x 128 for dx (174 a lane, 512 hold two).  Such a product waits for C to be written: 4 x 2048 x 64 -> 8192 bf16 41 us without, with
// it 35; 15 x 2120 x 16 -> 4096 120 and 84.  (Counted for dx too, as it was: 4 x 2048 x 8192 from 100 outputs 63.5 us, now 52.9, 8 x 2048 x 2048 from 40 30.9
// and 26.8; of eight such sizes 15 x 2120 x 4096 from 64 alone lost, 85 and 91.)
inline bool short_k(int64_t k, int bytes) { return k < 2 * kRowBytes / bytes; }

// The tile and the parts of k of the least cost.  Parts cost a second kernel and their sums' way through memory.
inline Plan gemm_plan(int learners, int64_t m, int64_t n, int64_t k, int bytes, int cus, bool dx = false) {
    Plan best{64, 64, 1};
    if (m < 1 || n < 1) return best;          // nothing to multiply
    const int64_t steps = parts_of(k, kRowBytes / bytes);
    float least = INFINITY;
    const TileCost* const costs = bytes == 4 ? kCostsFloat : kCostsBf16;
    for (const TileCost* at = costs; at < costs + (bytes == 4 ? std::size(kCostsFloat) : std::size(kCostsBf16)); ++at) {
        const TileCost& c = *at;
        const int64_t tiles = parts_of(m, c.rows) * parts_of(n, c.cols) * learners;
        const bool one_more = short_k(k, bytes) && c.resident > 1 && !(dx && c.rows == 128 && c.cols == 128);
        for (int split : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (split > 1 && (steps < 2 * split || tiles * split > 8 * (int64_t)cus)) break;
            const int64_t groups = tiles * split, each = parts_of(steps, split), room = (int64_t)cus * (c.resident + one_more);
            const float deep = (float)parts_of(groups, cus), rounds = (float)parts_of(groups, room);
            const float step = groups <= room ? (deep * c.shared > c.alone ? deep * c.shared : c.alone) : deep * c.shared;
            float us = (float)each * step + rounds * c.ends;
            if (split > 1) us += 4.0f + (float)(split + 1) * (float)(m * n * learners) * 4.0f / 3.5e6f;
            if (us < least) {
                least = us;
                best = Plan{c.rows, c.cols, split};
            }
        }
    }
    return best;
}

// Four outputs a wavefront where that leaves eight wavefronts for each compute unit.
inline bool four_outputs(int learners, int64_t out, int cus) { return out * learners >= (int64_t)cus * 32; }
// Tokens that few_tokens_kernel takes: no tiles then, and no parts of k.  us, this kernel / tiles: float 1 token 4096 x 4096 12 / 19, of eight learners
// 97 / 125, 4 tokens of eight learners 106 / 131; 8 tokens with an output a wavefront 4 x 1024 x 1024 7 / 12, with four 16 x 4489 x 4696 324 / 291 and
// 16 x 4096 x 2048 125 / 126; bf16 1 token 4096 x 4096 5 / 12, 4 tokens 8 / 13 and of sixteen learners, 4489 x 4696, 165 / 235.
inline int most_few(int learners, int64_t out, int bytes, int cus) { return bytes == 2 || four_outputs(learners, out, cus) ? 4 : 8; }
inline Plan forward_plan(int learners, int64_t t, int64_t out, int64_t in, int bytes, int cus) {
    return t <= most_few(learners, out, bytes, cus) ? Plan{64, 64, 1} : gemm_plan(learners, t, out, in, bytes, cus);
}

// ------------------------------------------------------------------------------------------------ its gradients
inline int64_t slope_slabs(int learners, int64_t t, int64_t o, int bytes, int cus) {
    const int64_t across = parts_of(o, kWave * 16 / bytes) * learners;
    if (across < 1) return 1;
    int64_t slabs = parts_of((int64_t)cus * 4, across);
    if (slabs > parts_of(t, 16)) slabs = parts_of(t, 16);
    return slabs < 1 ? 1 : slabs > 65535 ? 65535 : slabs;
}

// Whether few_tokens_grad_kernel makes dW.  us, it / tiles: 4 tokens of eight learners 6400 x 4096 float 155 / 282, bf16 86 / 144, of one 4096 x 4096
// 13 / 25 and 10 / 15; 16 float tokens 167 / 282 and 19 / 25, 8 bf16 92 / 145 and 14 / 16.
inline bool few_tokens_grad(int64_t t, int64_t out, int bytes) { return t >= 1 && t <= (bytes == 2 ? 8 : 16) && out < 1 << 24; }

struct GradRoom {
    size_t dz, sums, product, total;
    int64_t dz_pitch;
};
inline GradRoom grad_room(int act, int learners, int64_t t, int64_t in, int64_t out, int bytes, int cus, bool dx, bool dw, bool db) {
    GradRoom r{};
    r.dz_pitch = parts_of(out, 16 / bytes) * (16 / bytes);
    r.dz = act != PSGD_ACT_NONE ? up256((size_t)learners * t * r.dz_pitch * bytes) : 0;
    r.sums = db ? up256((size_t)learners * slope_slabs(learners, t, out, bytes, cus) * out * sizeof(float)) : 0;
    const size_t a = dx ? gemm_plan(learners, t, in, out, bytes, cus, true).bytes(learners, t, in) : 0;
    const size_t b = dw && !few_tokens_grad(t, out, bytes) ? gemm_plan(learners, out, in, t, bytes, cus).bytes(learners, out, in) : 0;
    r.product = a > b ? a : b;
    r.total = r.dz + r.sums + r.product;
    return r;
}

// The launches of the two products: one for both, or dx's and dW's, which for a few tokens is few_tokens_grad_kernel's.
struct GradPlan {
    Plan dx, dw;
    bool pair, few;
    int few_rows;          // of dW to a wavefront there
};
inline GradPlan grad_plan(int learners, int64_t t, int64_t in, int64_t out, int bytes, int cus, bool dx, bool dw) {
    GradPlan g{gemm_plan(learners, t, in, out, bytes, cus, true), gemm_plan(learners, out, in, t, bytes, cus), false, few_tokens_grad(t, out, bytes), 0};
    // one launch for both, also of few tokens where dW is small: 8192 x 500 bf16, 4 tokens, 9.6 us, apart 7.4 and 6.6
    const bool small = (int64_t)learners * in * out * bytes <= (8 << 20);
    g.pair = dx && dw && (!g.few || small) && g.dx.split == 1 && g.dw.split == 1 && g.dx.rows == g.dx.cols && g.dx.rows == g.dw.rows &&
             g.dw.rows == g.dw.cols && g.dx.rows < (bytes == 4 ? 128 : 256) &&       // (no two float products choose 128 x 128 together)
             (parts_of(t, g.dx.rows) * parts_of(in, g.dx.rows) + parts_of(out, g.dx.rows) * parts_of(in, g.dx.rows)) * learners <= kMostGroups;
    // 64 rows a wavefront, fewer where that leaves compute units without eight wavefronts
    const int64_t all = parts_of(in, kWave * 16 / bytes) * learners * out;
    g.few_rows = all >= (int64_t)cus * 8 * 64 ? 64 : all >= (int64_t)cus * 8 * 16 ? 16 : 4;
    return g;
}

// ------------------------------------------------------------------------------------------------ losses
constexpr int kUnroll = 4;               // 16-byte groups a lane has on their way: a batch

// Rows of a workgroup: one, or one for each of four wavefronts.
constexpr int rows_of_group(int lanes) { return lanes == kWave ? 4 : 1; }

// Lanes for a row.  us, k = 20, rows x columns, 64 / 256 / 1024 lanes: 64 000 x 500 bf16 88 / 266 / 3549; 3200 x 1000 float 11 / 15 / 41; 4096 x 32 000
// bf16 63 / 65 / 111, float 126 / 111 / 127; 4096 x 131 072 bf16 368 / 201 / 209; 256 x 200 000 float 288 / 105 / 66.  64 lanes have as many groups
// of lanes, of which the 33rd best and beyond are no good threshold.  (Cutting a few long rows into parts that a second kernel joins was no faster: the
// search's latency counts twice then.  1 x 131 072 bf16 20.5, uncut 16.9.)
inline int lanes_of_row(int64_t rows, int64_t groups, int k, int cus) {
    if (k <= 32 && (groups <= 256 || (groups <= 2048 && rows >= 4 * (int64_t)cus))) return 64;
    return groups <= 1024 || rows >= 4 * (int64_t)cus ? 256 : 1024;
}
// Bytes of batches' maxima that a workgroup keeps; rows with more (beyond 393 216 floats) have all batches looked at.
constexpr int batch_room(int lanes) { return lanes == 1024 ? 96 * 1024 : 40 * 1024; }
// Floats of LDS for a row's batches' maxima, 0 if they do not fit.
inline int batches_kept(int64_t groups, int lanes) {
    const int64_t floats = parts_of(groups, (int64_t)lanes * kUnroll) * lanes;
    return floats * rows_of_group(lanes) * 4 <= batch_room(lanes) ? (int)floats : 0;
}

// How distillation holds a row of so many 16-byte groups: so many lanes, `held` groups each; 0: none, the row is read again for the gradient.  Rows of
// 32 to 64 KB are held by 1024 lanes, two rows a compute unit at a time, or by 256 of sixteen groups each, four: the first are done with a row sooner, the
// second take half as many turns, which counts from the third row of a compute unit to about the eighth.  us, 1024 / 256 lanes:
//     rows                     512         520         1024        1536        2048        2560        4096
//     10 007 float          10.0 / 10.5  13.0 / 10.9  19.3 / 16.5  26.0 / 25.5  32.0 / 30.6  38.0 / 38.5  66.1 / 67.4
//     16 384 float          13.5 / 13.7  16.3 / 14.4  24.4 / 20.3  34.0 / 32.0  45.4 / 45.2  64.3 / 67.3   101 / 109
//     20 000 bf16           13.8 / 14.0  17.6 / 16.7  24.7 / 23.4  32.6 / 29.4  40.7 / 37.6  48.5 / 44.4  78.7 / 70.3
//     32 768 bf16           17.3 / 17.6  20.4 / 20.3  27.9 / 25.2  37.5 / 32.2  48.6 / 50.1  68.5 / 70.1   104 / 113
struct DistillHold {
    int lanes, held;
};
inline DistillHold distill_hold(int64_t rows, int64_t groups, bool gradient, int cus) {
    if (!gradient) return {groups <= 256 ? 64 : groups <= 256 * 16 ? 256 : 1024, 0};
    if (groups <= 64) return {64, 1};
    if (groups <= 64 * 2) return {64, 2};
    if (groups <= 64 * 4) return {64, 4};
    if (groups <= 256 * 2) return {256, 2};
    if (groups <= 256 * 4) return {256, 4};
    if (groups <= 256 * 8) return {256, 8};
    if (groups <= 256 * 16 && rows > 2 * (int64_t)cus && rows <= 8 * (int64_t)cus) return {256, 16};
    if (groups <= 1024 * 4) return {1024, 4};
    if (groups <= 1024 * 8) return {1024, 8};
    if (groups <= 1024 * 16) return {1024, 16};
    return {1024, 0};
}

}  // namespace psgd
#endif
