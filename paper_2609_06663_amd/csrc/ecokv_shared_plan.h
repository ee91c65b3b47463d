// How ecokv_decode_shared splits a call over blocks, and where a paged row
// lies: the arithmetic that the workspace size, the grid and the kernels share.
// Values only, no device state, so that it can be evaluated on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "ecokv.h"

namespace ecokv {

constexpr int kShWaves = 4;                     // waves per block
constexpr int kShTile = 32;                     // rows a wave takes at a time (fp32: 16)
constexpr int kShStep = kShWaves * kShTile;     // a part's rows are a multiple of this
constexpr int kShBlocks = 512;                  // blocks that fill the device

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

// Rows of one of `parts` equal parts of n rows, and how many parts have rows.
__host__ __device__ inline int64_t part_rows(int n, int parts)
{
    const int64_t r = ((int64_t)n + parts - 1) / parts;
    return (r + kShStep - 1) / kShStep * kShStep;
}
__host__ __device__ inline int parts_used(int n, int parts)
{
    return n > 0 ? (int)((n + part_rows(n, parts) - 1) / part_rows(n, parts)) : 0;
}

// A call's blocks.  The prompt's part: for each (layer, KV head), prompt and
// tile of `qt` query rows (G x its continuations), np parts of the kept rows.
// The tails' part: for each (layer, KV head), continuation and 16 query heads,
// nt parts of the tail.  Each block writes a partial of each of its query rows
// to the part's place in the workspace: [np + nt][L H_q N] sums [D], and
// (maximum, sum).
struct SharedGrid {
    int qt;              // query rows of a prompt block
    int np, nt;          // parts per unit of kept rows and per tail
    int tiles;           // query tiles of the prompts of a (layer, KV head)
    int tile0[ECOKV_MAX_SEQS + 1];  // before each prompt
    int64_t prompt_blocks, tail_blocks, qrows;
    size_t bytes;
};
__host__ __device__ inline int tail_groups(int G) { return (G + 15) / 16; }

inline int parts_for(int64_t blocks, int rows)
{
    const int64_t want = blocks > 0 ? (kShBlocks + blocks - 1) / blocks : 1, most = ((int64_t)rows + kShStep - 1) / kShStep;
    return (int)(rows <= 0 ? 0 : want < most ? want : most);
}

inline SharedGrid shared_grid(int64_t pairs, int G, int D, int B, const int32_t *fan, int max_count, int max_tail)
{
    SharedGrid g{};
    const int N = fan[B];
    g.qt = 16;
    for (int s = 0; s < B; ++s)
        g.tile0[s + 1] = g.tile0[s] + (int)(((int64_t)G * (fan[s + 1] - fan[s]) + g.qt - 1) / g.qt);
    g.tiles = max_count > 0 ? g.tile0[B] : 0;
    g.np = parts_for(pairs * g.tiles, max_count);
    g.nt = parts_for(pairs * N * tail_groups(G), max_tail);
    g.prompt_blocks = pairs * g.tiles * g.np;
    g.tail_blocks = pairs * N * tail_groups(G) * g.nt;
    g.qrows = pairs * G * N;
    g.bytes = sizeof(float) * (size_t)(g.np + g.nt) * (size_t)g.qrows * (size_t)(D + 2);
    return g;
}

}  // namespace ecokv
