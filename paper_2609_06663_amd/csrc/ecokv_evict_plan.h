// How ecokv_accumulate and ecokv_evict split a call, and the size of an eviction's
// plan.  Values only, no device state, so that it can be evaluated on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace ecokv {

constexpr int kMassWaves = 4;   // waves per block
constexpr int kMassRows = 32;   // rows of a wave at a time

// Blocks of ecokv_accumulate: a block takes four waves' rows of a unit or a tail at a
// time.  Where there are more than kMassBlocks such pieces, it takes several of its
// unit's, `parts` apart: the queries are listed and staged once for all of them.  (Us,
// 28 layers of 6553 kept rows and four tails of 777, one query of each and accepted
// paths: a piece a block 59.7 and 85.0, 1536 blocks 49.0 and 75.0, twice as many 50.1 and
// 76.7, half as many 55.3 and 82.7; 64 rows of a wave and 1536 blocks 55.4 and 78.6.)
constexpr int kMassBlocks = 1536;
inline void mass_grid(int64_t pairs, int B, int conts, int max_count, int max_tail, int *kept_parts, int *tail_parts,
                      int64_t *kept_blocks, int64_t *tail_blocks)
{
    const auto pieces = [](int64_t rows, int64_t each) { return (rows + each - 1) / each; };
    const int64_t each = kMassRows * kMassWaves;
    const int64_t all = pairs * B * pieces(max_count, each) + pairs * conts * pieces(max_tail, each);
    const int64_t several = (all + kMassBlocks - 1) / kMassBlocks, s = several < 1 ? 1 : several > 8 ? 8 : several;
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
