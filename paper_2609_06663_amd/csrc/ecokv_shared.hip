// ecokv_decode_shared kernels (gfx950): one query of each continuation of a
// batch over its prompt's kept rows and its own paged tail.
//
// For a (layer, KV head) the query rows that read one prompt's rows are its G
// query heads of all the prompt's continuations: M = G n of them, so the rows
// are the operands of matrix products, read once for a tile of up to 128 query
// rows instead of once for every continuation.  Softmax over both sets of rows:
// each block takes a part of one set for one tile of query rows and leaves
// (maximum, sum, sum of weighted values); k_shared_merge joins a query row's
// partials by their log-sum-exp.
//
// A wave has 32 query rows (fp32: 16) and takes as many rows of the cache at a
// time, from LDS, where they are staged while the rows before them are used.
//  * S^T = K Q^T: the rows as A, the query rows as B (v_mfma_f32_32x32x16_bf16,
//    or v_mfma_f32_16x16x4_f32).  A lane holds the logits of one query row
//    against half (a quarter) of the rows.
//  * O^T += V^T P^T: the weights are the B operand in the registers they are
//    computed in, and V^T, read transposed from LDS, takes their order of rows.
//    Every lane's sums belong to its query row, whose maximum and sum it also
//    keeps, so moving the reference (lazily, when a tile exceeds it by more than
//    2^8) costs no exchange.
//  * bf16 rows: a weight enters the product as three bf16 summands, its 24 bits
//    cut in three: rounded to one it would keep 2^-9 of every weight, and two
//    2^-17, where the sums beside it are fp32.
#include "ecokv_shared_device.h"

namespace ecokv {

__device__ __forceinline__ void tail_item(const SharedArgs &a, uint32_t w, SharedItem &it)
{
    const SharedGrid &g = a.grid;
    const uint32_t e = w / (uint32_t)g.nt;
    const int part = (int)(w - e * (uint32_t)g.nt);
    const uint32_t f = g.groups == 1 ? e : e / (uint32_t)g.groups;
    const int z = (int)(e - f * (uint32_t)g.groups);
    const int lh = (int)(f / (uint32_t)a.N);
    it.c0 = (int)(f - (uint32_t)lh * (uint32_t)a.N);
    const int n = uniform_i32(a.tail_counts[it.c0]);
    it.nc = 1;
    it.q0 = z * kTailQ;
    it.nq = min(kTailQ, a.G - it.q0);
    it.l = (int)((uint32_t)lh / (uint32_t)a.Hkv);
    it.h = lh - it.l * a.Hkv;
    it.part = g.np + part;
    it.base = 0;
    item_rows(it, n, a.max_tail, g.nt, part, g.tail_step);
}

// A wave's part of a tail: rows in pages, a tile ahead in registers.
template <bool BF, int D>
__device__ __forceinline__ void tail_part(const SharedArgs &a, const SharedItem &it, u32x4s *stage)
{
    typedef ShGeo<BF, D, 16> Ge;
    const int lane = threadIdx.x & 63, seg = lane % Ge::S, rg = lane / Ge::S;
    // the page of this lane's row of a tile (row lane % TR; clamped to the last row), -1 for none
    const auto pages = [&](int t) { return tail_page(a.map, it.c0, it.row0 + min(t * Ge::TR + lane % Ge::TR, it.rows - 1)); };
    u32x4s ld[2 * Ge::NL];
    const auto load = [&](int t, int page) {
#pragma unroll
        for (int i = 0; i < Ge::NL; ++i) {
            const int r = Ge::RPI * i + rg;
            const int row = it.row0 + min(t * Ge::TR + r, it.rows - 1);
            const int64_t at = tail_row(a.map, a.Hkv, it.l, it.h, max(__shfl(page, r, kWave), 0), row) * Ge::RB + 16 * seg;
            ld[i] = *reinterpret_cast<const u32x4s *>(a.Kt + at);
            ld[Ge::NL + i] = *reinterpret_cast<const u32x4s *>(a.Vt + at);
        }
    };
    const int nt = (it.rows + Ge::TR - 1) / Ge::TR;
    int page = pages(0), next = pages(1);
    load(0, page);
    ShState<BF, D, 16> w;
    load_queries<BF, D, 16>(a, it, it.q0, it.nq, w);
    for (int t = 0; t < nt; ++t) {
        const int left = it.rows - t * Ge::TR;
        const unsigned bad = (unsigned)(__builtin_amdgcn_ballot_w64(page < 0) & ((1ull << Ge::TR) - 1));
#pragma unroll
        for (int i = 0; i < Ge::NL; ++i) {
            const int r = Ge::RPI * i + rg;
            stage[stage_chunk<BF, Ge::S>(r, seg)] = ld[i];
            // (a row that is not there may hold no infinity)
            stage[Ge::TILE + stage_chunk<BF, Ge::S>(r, seg)] = r < left ? ld[Ge::NL + i] : (u32x4s){0u, 0u, 0u, 0u};
        }
        page = next;
        load(t + 1, page);  // (past the end: the last row again)
        next = pages(t + 2);
        __builtin_amdgcn_sched_barrier(0);
        typename Ge::X x;  // (a wave's own LDS accesses are ordered)
        first_tile<BF, D, 16>(stage, x, [&](typename Ge::X &y, float &mb) { tile_mask<BF, D, 16>(y, mb, left, bad); }, a.qscale, w);
        tile_values<BF, D, 3>(stage + Ge::TILE, x, a.qscale, w);
    }
    write_partials<BF, D, 16>(a, it, it.q0, it.nq, w);
}

template <bool BF, int D, int WQ>
__global__ __launch_bounds__(kShThreads, 2) void k_shared(SharedArgs a)
{
    typedef ShGeo<BF, D, 16> Ge;
    __shared__ u32x4s lds[kShWaves * 2 * Ge::TILE];
    static_assert(sizeof lds >= kShWaves * (BF ? 32 : 16) * D * sizeof(float), "the stages and the waves' sums share LDS");
    const uint32_t b = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    const uint32_t prompts = (uint32_t)a.grid.prompt_blocks;
    SharedItem it;
    if (b < prompts) {
        // Each XCD takes a run of the prompts' work, in which the tiles of a part are
        // neighbours: its L2 reads their rows once (eight continuations of 6553 rows,
        // two tiles of each part, 18.0 -> 16.5 us).
        const uint32_t x = b % kShXcds, q = prompts / kShXcds, r = prompts % kShXcds;
        prompt_item(a, x * q + min(x, r) + b / kShXcds, it);
        if (it.rows > 0) prompt_part<BF, D, WQ, 3>(a, it, lds);
    } else {
        const int wv = uniform_i32(threadIdx.x >> 6);
        const uint32_t w = (b - prompts) * kShWaves + wv;
        if (w >= (uint32_t)a.grid.tail_waves) return;
        tail_item(a, w, it);
        if (it.rows > 0) tail_part<BF, D>(a, it, lds + wv * 2 * Ge::TILE);
    }
}

template <bool BF, int D>
static void launch_shared(const SharedArgs &a, dim3 grid, hipStream_t st)
{
    if (a.grid.wq == 4) hipLaunchKernelGGL((k_shared<BF, D, 4>), grid, dim3(kShThreads), 0, st, a);
    else if (a.grid.wq == 2) hipLaunchKernelGGL((k_shared<BF, D, 2>), grid, dim3(kShThreads), 0, st, a);
    else hipLaunchKernelGGL((k_shared<BF, D, 1>), grid, dim3(kShThreads), 0, st, a);
}

hipError_t shared_launch(SharedArgs a, bool bf16, hipStream_t st)
{
    const int64_t blocks = a.grid.prompt_blocks + (a.grid.tail_waves + kShWaves - 1) / kShWaves;
    if (blocks > 0) {
        const dim3 g = blocks_grid(blocks);
        if (bf16 && a.D == 128) ECOKV_TIMED("decode_shared", st, (launch_shared<true, 128>(a, g, st)));
        else if (bf16) ECOKV_TIMED("decode_shared", st, (launch_shared<true, 64>(a, g, st)));
        else if (a.D == 128) ECOKV_TIMED("decode_shared", st, (launch_shared<false, 128>(a, g, st)));
        else ECOKV_TIMED("decode_shared", st, (launch_shared<false, 64>(a, g, st)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return merge_launch<false>(a, st);
}

}  // namespace ecokv
