// Which kernel, tile and number of parts an attention call takes: plain host arithmetic on sizes, types and the number of compute units, kept apart from
// the kernels so that a CPU build can say what a size runs.
#ifndef PSGD_ATTENTION_PLAN_H
#define PSGD_ATTENTION_PLAN_H

#include <cstddef>
#include <cstdint>

#include "psgd_attention.h"
#include "psgd_layers_plan.h"

namespace psgd {

// A head's columns as the kernels hold them: the rest is zero.
inline int held_head(int head) { return head <= 64 ? 64 : head <= 128 ? 128 : 256; }

// Rows of a workgroup's own, a matrix instruction's 16 columns or two times that for each of its wavefronts, and rows of the tiles that it walks.
constexpr int kAttentionWaves = 4;
constexpr int own_blocks(int held, int bytes) { return bytes == 2 && held <= 128 ? 2 : 1; }
constexpr int own_rows(int held, int bytes) { return kAttentionWaves * 16 * own_blocks(held, bytes); }
constexpr int walked_rows(int held, int bytes) { return held * bytes <= 256 ? 64 : 32; }

// Places for the own tiles of a learner's sequences: sequence s has its from starts[s] / rows + s on, which leaves every sequence room for all of its
// tiles whatever their lengths, so that a workgroup finds its sequence by itself and no launch depends on device memory.
inline int64_t tile_places(int64_t t, int sequences, int rows) { return t / rows + (sequences > 0 ? sequences : 1); }

// ------------------------------------------------------------------------------------------------ one new token
constexpr int kStepWaves = 4;
constexpr int kStepKeys = 32;               // of a wavefront at a time
// Parts that a sequence's keys are cut into.
inline int step_parts(int64_t units, int64_t most_keys, int cus) {
    const int64_t most = parts_of(most_keys, kStepWaves * kStepKeys * 2), fair = parts_of((int64_t)cus * 4, units);
    const int64_t p = most < fair ? most : fair;
    return (int)(p < 1 ? 1 : p > 1024 ? 1024 : p);
}

}  // namespace psgd
#endif
