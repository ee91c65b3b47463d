// How ecokv_decode_shared splits a call over blocks, and where a paged row
// lies: the arithmetic that the workspace size, the grid and the kernels share.
// Values only, no device state, so that it can be evaluated on the host.
#pragma once

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "ecokv.h"

namespace ecokv {

constexpr int kShWaves = 4;                     // waves per block
constexpr int kShNarrow = 210 << 20;            // bytes (see shared_grid)
constexpr int kTailQ = 16;                      // query heads of a wave in the tails
constexpr int kShBlocks = 256;                  // compute units: blocks of one round (two fit a unit)
constexpr int kShMostRows = 1 << 22;            // rows of a part at most: its bytes are addressed by 32 bits

// The page of row `row` of continuation `cont`, or -1: a row outside the
// table, a continuation outside it, a page outside the pool.
struct TailMap {
    const int32_t *table;
    int conts, pages, shift, max_pages;
};
__host__ __device__ inline int tail_page(const TailMap &m, int cont, int row)
{
    if (cont < 0 || cont >= m.conts || row < 0 || (row >> m.shift) >= m.max_pages) return -1;
    const int p = m.table[(int64_t)cont * m.max_pages + (row >> m.shift)];
    return p >= 0 && p < m.pages ? p : -1;
}
// The row of the pool [L][pages][H_kv][page_size] that page `page`, layer l and
// KV head h have for row `row` of a tail.
__host__ __device__ inline int64_t tail_row(const TailMap &m, int Hkv, int l, int h, int page, int row)
{
    return ((((int64_t)l * m.pages + page) * Hkv + h) << m.shift) + (row & ((1 << m.shift) - 1));
}

// Rows of one of `parts` equal parts of n rows, a multiple of `step` (a power of
// two), and how many parts have rows.  (Unsigned: n plus what rounding adds may
// pass 2^31, and 32-bit divisions take a third of the time of 64-bit ones.)
__host__ __device__ inline uint32_t part_rows(int n, int parts, int step)
{
    const uint32_t r = ((uint32_t)n + (uint32_t)parts - 1u) / (uint32_t)parts;
    return (r + (uint32_t)step - 1u) & ~((uint32_t)step - 1u);
}
__host__ __device__ inline int parts_used(int n, int parts, int step)
{
    if (n <= 0) return 0;
    const uint32_t r = part_rows(n, parts, step);
    return (int)(((uint32_t)n + r - 1u) / r);
}

// A call's work.
//  * The prompt's part.  The query rows of a (layer, KV head) and prompt, G x
//    its continuations, are cut into tiles of wq x rows_q, rows_q per wave;
//    its kept rows into np parts.  A block takes one tile and one part; the
//    four waves' 4 / wq groups share the part's rows.
//  * The tails' part.  A wave takes kTailQ query heads of a (layer, KV head) and
//    continuation and one of nt parts of the tail; four waves share a block.
// Each leaves a partial of every query row at the part's place in the
// workspace: [np + nt][L H_q N] sums [D], and (maximum, sum).
// Rows are taken rows_t at a time; rows_q and rows_t are 32 (bf16) or 16 (fp32).
struct SharedGrid {
    int rows_q, rows_t, wq;
    int np, nt;               // parts of a unit's kept rows, of a tail
    int step, tail_step;      // a prompt part's and a tail part's rows are multiples of these
    int tiles;                // query tiles of the prompts of a (layer, KV head)
    int tile0[ECOKV_MAX_SEQS + 1];  // before each prompt
    int groups;               // groups of kTailQ query heads of a tail
    int64_t prompt_blocks, tail_waves, qrows;
    size_t bytes;
};

// Between the least and the most parts of `rows` rows: none of fewer than `step`
// rows or of more than kShMostRows.
inline int parts_within(int64_t parts, int rows, int step)
{
    const int64_t most = ((int64_t)rows + step - 1) / step, least = ((int64_t)rows + kShMostRows - 1) / kShMostRows;
    if (parts > most) parts = most;
    return (int)(parts < least ? least : parts);
}

// Parts of the prompts' rows for `have` (unit, tile)s.  As many as one round of
// blocks holds, if that is eight or more: every further part is a partial of each
// query row to write and to merge (us, one block per compute unit against two: 64
// continuations of 6553 rows 40 and 49, 20 of 64 heads of 8191 rows 39 and 43).
// With fewer, rounds may stay nearly empty, and 1 to 8 parts are weighed by the
// time they would take: rounds of blocks, each a start and its rows, beside the
// time of the rows' bytes, and the partials' bytes.  us, with the parts of one
// round and so chosen, 16 continuations of 6553 rows: 136 units of 4 heads 130 and
// 111, 160 132 and 123, 264 235 and 212, 320 250 and 236, 512 the same, 192 140 and
// 146; 112 units of 7 heads 124 and 118, 132 187 and 143, 256 263 and 241; fp32, 160
// units of 4 heads, 6 continuations of 2000 rows, 158 and 119.
inline int prompt_parts(const SharedGrid &g, int64_t have, int64_t units, int D, int rows, bool bf16)
{
    if (rows <= 0 || have <= 0) return 0;
    int64_t best = kShBlocks / have;
    if (best < 8) {
        // a block's row: one wave per row waits for memory, more for its products
        const double us = (bf16 ? (g.wq == 1 ? 0.013 : 0.0088 * g.wq) : 0.018 * g.wq) * D / 128;
        const double read = (double)units * rows * D * (bf16 ? 4 : 8) / 5.3e6, part = (double)g.qrows * (D + 2) * 8 / 2.6e6;
        double least = 0;
        best = 0;
        for (int np = 1; np <= 8; ++np) {
            const double rounds = (double)((have * np + kShBlocks - 1) / kShBlocks);
            // (two blocks of four waves per row overlap a little)
            double t = rounds * (rows * us / np + 3.5) / (g.wq == 4 && rounds > 1 ? 1.15 : 1.0);
            t = cbrt(t * t * t + read * read * read) + np * part;  // (neither hides behind the other wholly)
            if (best == 0 || t < least) best = np, least = t;
        }
    }
    return parts_within(best, rows, g.step);
}

// Parts of a tail for `have` waves: a wave for each of the four SIMDs of a
// compute unit; without prompts, whose blocks fill as many places, for two, where
// that gives up to four parts (us, with parts for one and for two, tails of 777
// rows: 400 units 40 and 34, 600 64 and 48, 800 80 and 65; beside prompts, 400 units
// 54 and 58, 256 40 and 43).
inline int tail_parts(bool alone, int64_t have, int rows, int step)
{
    if (rows <= 0 || have <= 0) return 0;
    const int64_t one = kShBlocks * kShWaves / have, two = 2 * kShBlocks * kShWaves / have;
    return parts_within(!alone || one > 4 ? one : two > 4 ? 4 : two, rows, step);
}

inline SharedGrid shared_grid(int64_t pairs, int G, int D, int B, const int32_t *fan, int max_count, int max_tail, bool bf16)
{
    SharedGrid g{};
    const int N = fan[B];
    g.rows_q = g.rows_t = bf16 ? 32 : 16;
    int64_t most = 0, tiles = 0, prompts = 0;  // query rows of the largest prompt; tiles of rows_q of all; prompts that have any
    for (int s = 0; s < B; ++s) {
        const int64_t m = (int64_t)G * (fan[s + 1] - fan[s]);
        most = m > most ? m : most;
        tiles += (m + g.rows_q - 1) / g.rows_q;
        prompts += m > 0;
    }
    // As many waves along the query rows as the largest prompt fills: each row of
    // the cache then serves them all from LDS.  But where the tiles of rows_q
    // together read no more than kShNarrow bytes, a block for each: the L2 of the
    // XCD that has all of a part's tiles bears that, more blocks share the rows'
    // latency, and no wave of a small prompt idles (us, wide and narrow: 14 tiles of
    // 6553 rows of 4 heads, 188 MB, 31.1 and 25.0; 4 layers of 4 such tiles, 215 MB,
    // 29.1 and 26.2; 4 tiles of 30000 rows, 246 MB, 28.5 and 31.2; 14 layers of 4
    // tiles of 6553, 752 MB, 59 and 67; fp32, 8 tiles of 6553, 215 MB, 29.3 and 29.5).
    const bool narrow = (double)(pairs * tiles) * max_count * D * (bf16 ? 4 : 8) <= (double)kShNarrow;
    g.wq = narrow ? 1 : most > 2 * g.rows_q ? 4 : most > g.rows_q ? 2 : 1;
    g.step = g.rows_t * (kShWaves / g.wq);
    g.tail_step = 2 * g.rows_t;
    const int qt = g.wq * g.rows_q;
    for (int s = 0; s < B; ++s) {
        g.tile0[s + 1] = g.tile0[s] + (int)(((int64_t)G * (fan[s + 1] - fan[s]) + qt - 1) / qt);
    }
    g.tiles = max_count > 0 ? g.tile0[B] : 0;
    g.groups = (G + kTailQ - 1) / kTailQ;
    g.qrows = pairs * G * N;
    g.np = prompt_parts(g, pairs * g.tiles, pairs * prompts, D, max_count, bf16);
    g.nt = tail_parts(g.np == 0, pairs * N * g.groups, max_tail, g.tail_step);
    g.prompt_blocks = pairs * g.tiles * g.np;
    g.tail_waves = pairs * N * g.groups * g.nt;
    g.bytes = sizeof(float) * (size_t)(g.np + g.nt) * (size_t)g.qrows * (size_t)(D + 2);
    return g;
}

}  // namespace ecokv
