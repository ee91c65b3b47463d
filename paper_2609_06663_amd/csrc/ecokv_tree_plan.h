// How ecokv_decode_tree splits a call over blocks: the arithmetic that the
// workspace size, the grid and the kernels share.  Values only, as
// ecokv_shared_plan.h, whose prompt parts it takes.
#pragma once

#include "ecokv_shared_plan.h"

namespace ecokv {

// The tails' part of a call.  A continuation has nodes x G query rows for every
// (layer, KV head): cut into tiles of wq x rows_q; its tail and the drafted rows
// behind it into grid.nt parts.  wq = 4: a block takes one tile and one part;
// wq = 1: a wave does.  Part k has the rows from k * rows on, whatever the count.
struct TreeTails {
    int wq, tiles, rows;
    int64_t blocks;
};

// Several prompts' parts go by their counts, which the device alone knows (fill = 0:
// they do not).  All blocks work out the same length of a part in steps of two tiles:
// what gives about `fill` blocks, but between `least` and grid.np parts of the longest
// unit.  The grid holds the most blocks that this can be.  Some then have nothing to do,
// and the tails' blocks, which would wait for these, come first where their parts are
// not short beside the prompts' (ahead).  (us, 13 nodes of 5, 1 and 6 continuations with
// tails of 333 rows, 8 KV heads: equal parts, by counts, and the tails first: prompts of
// 4480, 619 and 2610 rows whose heads kept 6 to 14 tenths of them 44.9 39.8 36.0, three of
// 4480 so kept 49.9 45.0 44.1, wholly kept 42.0 43.7 43.6; 38 64-wide heads of 4441 and 2321
// rows, 18 and 4 answers of 265 68.7 59.6 74.7.)
struct TreeEven {
    int least, fill, ahead;
};
constexpr int kEvenUnits = 256;   // at most: four of a lane
constexpr size_t kEvenBytes = 16;  // of the workspace, behind the partials: a part's length

// Rows of a prompt's part that are worth a block of its own, in wide and in narrow
// tiles (us, 28 query rows of 4 heads, 1500 kept rows in parts of 768, 384 and 256: 15.7
// 13.6 13.7; 6553 in parts of 640, 480 and 384: 15.5 14.7 14.5).
constexpr int kTreeRows = 512, kTreeNarrowRows = 256;

// fan counts nodes (fan[s + 1] - fan[s] of prompt s); conts continuations.
inline SharedGrid tree_grid(int64_t pairs, int G, int D, int B, const int32_t *fan, int conts, int nodes, int max_count,
                            int max_tail, bool bf16, TreeTails *tails, TreeEven *even)
{
    SharedGrid g{};
    *tails = TreeTails{};
    *even = TreeEven{0, 0, 0};
    if (pairs <= 0 || conts <= 0) return g;  // (no layers, or nobody continues)
    g.rows_q = g.rows_t = bf16 ? 32 : 16;
    int64_t most = 0, narrow_tiles = 0, prompts = 0;
    for (int s = 0; s < B; ++s) {
        const int64_t m = (int64_t)G * (fan[s + 1] - fan[s]);
        most = m > most ? m : most;
        narrow_tiles += (m + g.rows_q - 1) / g.rows_q;
        prompts += m > 0;
    }
    // (as in shared_grid, but with query tiles of one wave or four)
    const bool narrow = (double)(pairs * narrow_tiles) * max_count * D * (bf16 ? 4 : 8) <= (double)kShNarrow;
    g.wq = narrow || most <= g.rows_q ? 1 : 4;
    g.step = g.rows_t * (kShWaves / g.wq);
    const int qt = g.wq * g.rows_q;
    for (int s = 0; s < B; ++s) g.tile0[s + 1] = g.tile0[s] + (int)(((int64_t)G * (fan[s + 1] - fan[s]) + qt - 1) / qt);
    g.tiles = max_count > 0 ? g.tile0[B] : 0;
    g.qrows = pairs * G * fan[B];
    const int rows = max_tail + nodes;
    const int64_t short_parts = ((int64_t)rows + 4 * g.rows_t - 1) / (4 * g.rows_t);  // of four tiles
    // A wave of its own for query rows that fit one, but not with 128-wide bf16 rows: its
    // loads, tile and sums need 62 registers more than there are (us, four waves and one:
    // 28 query rows of 4 heads and 704 rows 14.7 23.6, 28 layers of them 87 110, 8 layers of
    // 8000 rows 52 63; 128 heads of 24 query rows and 4000 rows 86 95; 64-wide, 1000 rows
    // 25.0 20.7, 8000 rows 103 65; fp32 of 6 such answers, 28 layers, 1000 rows 154 96).
    tails->wq = nodes * G <= g.rows_q && !(bf16 && D == 128) ? 1 : 4;
    const int tt = tails->wq * g.rows_q;
    tails->tiles = (nodes * G + tt - 1) / tt;
    const int64_t have = pairs * conts * tails->tiles;  // (continuation, tile)s
    const int64_t slots = 2 * kShBlocks;                // blocks that run at once
    const int64_t prompt_have = pairs * g.tiles, tail_least = tails->wq == 1 ? (have + kShWaves - 1) / kShWaves : have;

    g.np = prompt_parts(g, prompt_have, pairs * prompts, D, max_count, bf16);
    if (g.wq == 1 && g.np > 0) {
        // no shorter parts, and no block that shares its compute unit with a tail's,
        // where that takes few parts away (us, 112 query rows of 4 heads, 6553 kept rows,
        // 12 and 16 parts beside 24 blocks of tails: 20.2 23.0)
        const int64_t most = ((int64_t)max_count + kTreeNarrowRows - 1) / kTreeNarrowRows;
        const int64_t room = (kShBlocks - tail_least * short_parts) / prompt_have;
        int64_t np = g.np < most ? g.np : most;
        if (room < np && 4 * room >= 3 * np) np = room;
        g.np = parts_within(np, max_count, g.step);
    } else if (g.np > 0) {
        // two blocks per compute unit where the parts stay long
        const int64_t fill = (slots - tail_least) / prompt_have, most = max_count / kTreeRows;
        const int64_t np = fill < most ? fill : most;
        if (np > g.np) g.np = parts_within(np, max_count, g.step);
    }
    g.prompt_blocks = prompt_have * g.np;
    if (tails->wq == 1) {
        // waves: one for each SIMD, or two while their parts stay long
        g.tail_step = 2 * g.rows_t;
        const int64_t one = kShBlocks * kShWaves / have, two = 2 * kShBlocks * kShWaves / have;
        g.nt = parts_within(two > one && rows / two >= 256 ? two : one < 1 ? 1 : one, rows, g.tail_step);
    } else {
        // as many as there is room for beside the prompts, none short, and none longer
        // than a prompt's part (nor cut where that is short: 22 tails of 1810 rows beside
        // 22 x 76 kept rows took 100 us in 24 parts, 50 in 4)
        g.tail_step = 2 * g.rows_t;
        int64_t nt;
        if (g.np > 0) {
            int64_t like = ((int64_t)max_count + g.np - 1) / g.np;
            like = like < kTreeRows ? kTreeRows : like;
            const int64_t least = (rows + like - 1) / like;
            const int64_t room = (slots - g.prompt_blocks) / have;
            nt = room < short_parts ? room : short_parts;
            nt = nt > least ? nt : least;
        } else {
            nt = prompt_parts(g, have, pairs * conts, D, rows, bf16);
        }
        g.nt = parts_within(nt < 1 ? 1 : nt, rows, g.tail_step);
    }
    tails->rows = (int)part_rows(rows, g.nt, g.tail_step);
    g.nt = parts_used(rows, g.nt, g.tail_step);  // (rounded up, fewer may do)
    g.tail_waves = tails->wq == 1 ? have * g.nt : 0;
    tails->blocks = tails->wq == 1 ? (g.tail_waves + kShWaves - 1) / kShWaves : have * g.nt;
    if (g.wq == 4 && g.np > 0 && prompts > 1 && pairs * B <= kEvenUnits && g.prompt_blocks + tails->blocks <= slots) {
        const int64_t most = max_count / kTreeNarrowRows, twice = 2 * (int64_t)g.np;
        even->least = g.np;
        even->fill = (int)(slots - tails->blocks);
        g.np = parts_within(most < g.np ? g.np : most < twice ? most : twice, max_count, g.step);
        g.prompt_blocks = even->fill + prompt_have;
        even->ahead = 3 * (int64_t)tails->rows * even->fill >= prompt_have * max_count;
    }
    g.bytes = sizeof(float) * (size_t)(g.np + g.nt) * (size_t)g.qrows * (size_t)(D + 2) + (even->fill ? kEvenBytes : 0);
    return g;
}

}  // namespace ecokv
