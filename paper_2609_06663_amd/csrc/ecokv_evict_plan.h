// How ecokv_accumulate and ecokv_evict split a call, and the size of an eviction's
// plan.  Values only, no device state, so that it can be evaluated on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace ecokv {

constexpr int kMassWaves = 4;  // waves per block

// Blocks of ecokv_accumulate: a wave takes rt tiles of 16 rows of a unit or a tail at a
// time, a block four waves.  Where there are more than kMassBlocks such pieces, a block
// takes several of its unit's, `parts` apart: the queries are listed once for all of them
// (accepted paths of four continuations, 28 layers of 6553 kept rows, us: a piece a block
// 100, three 78).
constexpr int kMassBlocks = 1536;
inline void mass_grid(int64_t pairs, int B, int conts, int max_count, int max_tail, int *rt, int *kept_parts, int *tail_parts,
                      int64_t *kept_blocks, int64_t *tail_blocks)
{
    const auto pieces = [](int64_t rows, int64_t each) { return (rows + each - 1) / each; };
    const auto all = [&](int64_t each) { return pairs * B * pieces(max_count, each) + pairs * conts * pieces(max_tail, each); };
    *rt = all(64 * kMassWaves) >= 1024 ? 4 : 2;
    const int each = 16 * *rt * kMassWaves;
    const int64_t several = (all(each) + kMassBlocks - 1) / kMassBlocks, s = several < 1 ? 1 : several > 8 ? 8 : several;
    *kept_parts = (int)pieces(max_count, each * s);
    *tail_parts = conts > 0 ? (int)pieces(max_tail, each * s) : 0;
    *kept_blocks = pairs * B * *kept_parts;
    *tail_blocks = pairs * conts * *tail_parts;
}

// Words of a unit's plan: a head, and two for every row that may move to the place
// of an evicted one, no more than stay and no more than go.
constexpr int kPlanHead = 4;
inline int evict_plan_cap(int max_rows, int keep)
{
    const int go = max_rows - keep;
    return go < 0 ? 0 : go < keep ? go : keep;
}
inline int64_t evict_plan_words(int max_rows, int keep) { return kPlanHead + 2 * (int64_t)evict_plan_cap(max_rows, keep); }

}  // namespace ecokv
