// How ecokv_accumulate and ecokv_evict split a call, and the size of an eviction's
// plan.  Values only, no device state, so that it can be evaluated on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace ecokv {

constexpr int kMassWaves = 4;  // waves per block

// Blocks of ecokv_accumulate: a wave has rt tiles of 16 rows of a unit or a tail, a
// block four waves.
inline void mass_grid(int64_t pairs, int B, int conts, int max_count, int max_tail, int *rt, int *kept_parts, int *tail_parts,
                      int64_t *kept_blocks, int64_t *tail_blocks)
{
    const auto parts = [](int64_t rows, int each) { return (int)((rows + each - 1) / each); };
    const int64_t blocks = pairs * B * parts(max_count, 64 * kMassWaves) + pairs * conts * parts(max_tail, 64 * kMassWaves);
    *rt = blocks >= 1024 ? 4 : 2;
    const int each = 16 * *rt * kMassWaves;
    *kept_parts = parts(max_count, each);
    *tail_parts = conts > 0 ? parts(max_tail, each) : 0;
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
