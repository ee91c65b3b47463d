// ecokv_decode_tree kernels (gfx950): a tree of drafted tokens of every
// continuation over its prompt's kept rows, its paged tail and the drafted rows
// behind it.
//
// A prompt's kept rows are read by nodes x continuations x G query rows of a
// (layer, KV head): that part is ecokv_decode_shared's, a node in the place of a
// continuation (prompt_part).  A continuation's tail and drafted rows are read by
// its nodes x G query rows: the same tiles, rows found page by page.  Node i sees
// drafted row j where bit j of its mask is set, so a lane, which has one query
// row, masks the logits of its node; only tiles with drafted rows (or the last
// rows) are masked at all.  Partials are joined by k_shared_merge.
//
// What a node does not see must not reach it: logits are replaced, not weighed,
// and a drafted row that no node sees is staged as zeros.  One that some nodes see
// may hold an infinity or a NaN among its values, and 0 times that is NaN: such
// elements are staged as zeros too, remembered, and added to the partials of the
// nodes that see them afterwards.
#include "ecokv_shared_device.h"

namespace ecokv {

constexpr int kTreeSummands = 2;  // of a weight in the product with bf16 values

// Drafted rows of a part that need more than the loop does: no page there, or
// values that are not finite; and whether a tail row has no page.
struct TreeFlags {
    unsigned bad[2], poison[2], lost;
};

struct TreeItem : SharedItem {
    int c, n;  // continuation, its tail's rows
};

__device__ __forceinline__ void tree_item(const TreeArgs &a, uint32_t w, TreeItem &it)
{
    const SharedGrid &g = a.s.grid;
    const uint32_t e = w / (uint32_t)a.tails.tiles;
    const int z = (int)(w - e * (uint32_t)a.tails.tiles);
    const uint32_t f = e / (uint32_t)g.nt;
    const int part = (int)(e - f * (uint32_t)g.nt);
    const int lh = (int)(f / (uint32_t)a.conts);
    it.c = (int)(f - (uint32_t)lh * (uint32_t)a.conts);
    const int n = uniform_i32(a.s.tail_counts[it.c]);
    const bool valid = n >= 0 && n <= a.s.max_tail;
    const int qt = a.tails.wq * g.rows_q;
    it.n = n;
    it.c0 = it.c * a.s.nodes;
    it.nc = a.s.nodes;
    it.q0 = z * qt;
    it.nq = min(qt, a.s.G * a.s.nodes - it.q0);
    it.l = (int)((uint32_t)lh / (uint32_t)a.s.Hkv);
    it.h = lh - it.l * a.s.Hkv;
    it.part = g.np + part;
    it.base = 0;
    item_rows(it, valid ? n + a.s.nodes : 0, a.s.max_tail + a.s.nodes, g.nt, part, g.tail_step);
}

// What lanes of a wave wrote to LDS before is what others read after.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

template <bool BF>
__device__ __forceinline__ bool not_finite(uint32_t x)  // (bf16: either half)
{
    if constexpr (BF) return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
    else return (x & 0x7f800000u) == 0x7f800000u;
}
// x with zeros in the place of what is not finite.
template <bool BF>
__device__ __forceinline__ uint32_t finite_part(uint32_t x)
{
    if constexpr (BF) {
        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
        return x;
    } else {
        return not_finite<BF>(x) ? 0u : x;
    }
}

// Adds the drafted rows' values that are not finite to the partials of the query
// rows that see them: each lane to the sums that it wrote.
template <bool BF, int D, int QT>
__device__ __forceinline__ void add_poison(const TreeArgs &a, const TreeItem &it, int q0, int nq, unsigned long long sees,
                                        unsigned long long poison, float m)
{
    typedef ShGeo<BF, D, QT> Ge;
    const int lane = threadIdx.x & 63, q = lane % QT;
    if (q >= nq) return;
    const int row = q0 + q, g = row / it.nc, c = it.c0 + row % it.nc;
    const char *qp = a.s.Q + (((int64_t)it.l * a.s.Hq + it.h * a.s.G + g) * a.s.N + c) * Ge::RB;
    float *acc = a.s.acc + partial_row(a.s, it, row) * D;
    const auto at = [](const char *p, int d) {
        if constexpr (BF) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[d] << 16);
        else return reinterpret_cast<const float *>(p)[d];
    };
    for (unsigned long long left = poison & sees; left; left &= left - 1) {
        const int r = it.n + __ffsll(left) - 1;
        const int page = tail_page(a.s.map, it.c, r);
        const int64_t off = tail_row(a.s.map, a.s.Hkv, it.l, it.h, max(page, 0), r) * Ge::RB;
        float x = 0.f;
#pragma unroll 1
        for (int d = 0; d < D; ++d) x = fmaf(at(qp, d), at(a.s.Kt + off, d), x);
        const float p = exp2f(fmaf(x, a.s.qscale, m == -INFINITY ? 0.f : -m));
#pragma unroll 1
        for (int k = 0; k < Ge::DT * Ge::AX; ++k) {
            const int dim = sum_dim<QT>(k / Ge::AX, k % Ge::AX / 4) + k % 4;
            const float v = at(a.s.Vt + off, dim);
            if (!(fabsf(v) < INFINITY)) acc[dim] += p * v;
        }
    }
}

// A part of a tail and the drafted rows behind it for one tile of query rows, by
// the four waves of a block (WQ = 4) or by one wave (WQ = 1).
template <bool BF, int D, int WQ>
__device__ __forceinline__ void tree_part(const TreeArgs &a, const TreeItem &it, u32x4s *stage, TreeFlags *flags)
{
    constexpr int QT = BF ? 32 : 16, NS = BF ? kTreeSummands : 3;
    typedef ShGeo<BF, D, QT> Ge;
    constexpr int TR = Ge::TR, LPT = 2 * Ge::NL / WQ;  // load instructions of a wave for a tile
    const int lane = threadIdx.x & 63, wq = WQ == 1 ? 0 : uniform_i32(threadIdx.x >> 6);
    const int seg = lane % Ge::S, rg = lane / Ge::S;
    const int M = a.s.nodes, q0 = it.q0 + wq * QT, nq = min(it.nq - wq * QT, QT);
    const int first = it.n - it.row0;  // of the drafted rows, among the part's
    const bool drafted = first < it.rows;

    // what this lane's node sees of the drafted rows, and what any node does
    unsigned long long sees = 0, any = 0;
    if (drafted) {
        const unsigned long long within = M < 64 ? (1ull << M) - 1 : ~0ull;
        const int m = nq > 0 ? q0 + min(lane % QT, nq - 1) : it.q0;
        sees = a.masks[(int64_t)it.c0 + m % M] & within;
        any = lane < M ? a.masks[(int64_t)it.c0 + lane] & within : 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) any |= __shfl_xor(any, o, kWave);
    }
    if (WQ == 1 || threadIdx.x == 0) *flags = TreeFlags{};
    if constexpr (WQ == 1) wave_lds_order();

    // the page of this lane's row of a tile (row lane % TR; clamped to the last row), -1 for none
    const auto pages = [&](int t) { return tail_page(a.s.map, it.c, it.row0 + min(t * TR + lane % TR, it.rows - 1)); };
    const auto note = [&](int t, int page) {  // rows that have none
        if (__builtin_amdgcn_ballot_w64(page < 0)) {
            const int r = t * TR + lane;
            if (page < 0 && lane < TR && r < it.rows) {
                if (r < first) flags->lost = 1;
                else atomicOr(&flags->bad[(r - first) >> 5], 1u << ((r - first) & 31));
            }
        }
    };
    // instruction i of tile t; bit i of ok: the row is there
    const auto load = [&](const char *base, int i, int t, int page, u32x4s &x, unsigned &ok, int bit) {
        const int r = t * TR + Ge::RPI * i + rg, pg = __shfl(page, Ge::RPI * i + rg, kWave);
        const int row = it.row0 + min(r, it.rows - 1);
        x = *reinterpret_cast<const u32x4s *>(base + tail_row(a.s.map, a.s.Hkv, it.l, it.h, max(pg, 0), row) * Ge::RB + 16 * seg);
        const bool there = pg >= 0 && r < it.rows && (r < first || ((any >> (r - first)) & 1));
        ok = there ? ok | (1u << bit) : ok & ~(1u << bit);
    };
    const auto put_value = [&](u32x4s x, bool ok, int i, int t, u32x4s *to) {
        if (!ok) x = (u32x4s){0u, 0u, 0u, 0u};
        const int r = t * TR + Ge::RPI * i + rg;
        if (t * TR + TR > first) {
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = odd || not_finite<BF>(x[e]);
            if (odd && r >= first) {
                atomicOr(&flags->poison[(r - first) >> 5], 1u << ((r - first) & 31));
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = finite_part<BF>(x[e]);
            }
        }
        to[stage_chunk<BF, Ge::S>(Ge::RPI * i + rg, seg)] = x;
    };
    const auto mask = [&](int t) {
        return [&, t](typename Ge::X &x, float &mb) {
            const int left = it.rows - t * TR, d = first - t * TR;
            if (left < TR || d < TR) {
                __builtin_amdgcn_sched_barrier(0);
                const unsigned long long m = d >= 0 ? sees << min(d, 63) : -d < 64 ? sees >> -d : 0ull;
                unsigned v = (unsigned)m | (d >= 32 ? ~0u : d > 0 ? (1u << d) - 1u : 0u);
                if (left < 32) v &= left > 0 ? (1u << left) - 1u : 0u;
                mb = -INFINITY;
#pragma unroll
                for (int r = 0; r < Ge::NX; ++r) {
                    if (!((v >> tile_key<BF, D, QT>(r)) & 1u)) x[r] = -INFINITY;
                    mb = fmaxf(mb, x[r]);
                }
            }
        };
    };

    ShState<BF, D, QT> w;
    const int tiles = (it.rows + TR - 1) / TR;
    typename Ge::X x, y;
    if constexpr (WQ == 1) {
        // K a tile ahead of V, as in prompt_part
        u32x4s kx[Ge::NL], vx[Ge::NL];
        unsigned ok = 0, none = 0;
        int p0 = pages(0), p1 = pages(1), p2 = pages(2);
        {
            u32x4s k0[Ge::NL];
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) load(a.s.Kt, i, 0, p0, k0[i], none, i);
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) load(a.s.Kt, i, 1, p1, kx[i], none, i);
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) load(a.s.Vt, i, 0, p0, vx[i], ok, i);
            load_queries<BF, D, QT>(a.s, it, q0, nq, w);
            note(0, p0);
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) stage[stage_chunk<BF, Ge::S>(Ge::RPI * i + rg, seg)] = k0[i];
        }
        first_tile<BF, D, QT>(stage, x, mask(0), a.s.qscale, w);
        for (int t = 0; t < tiles; ++t) {
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) {
                stage[stage_chunk<BF, Ge::S>(Ge::RPI * i + rg, seg)] = kx[i];
                put_value(vx[i], (ok >> i) & 1u, i, t, stage + Ge::TILE);
            }
            note(t + 1, p1);
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) load(a.s.Kt, i, t + 2, p2, kx[i], none, i);
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) load(a.s.Vt, i, t + 1, p1, vx[i], ok, i);
            p1 = p2;
            p2 = pages(t + 3);
            __builtin_amdgcn_sched_barrier(0);
            tile_step<BF, D, QT, NS>(stage, stage + Ge::TILE, x, y, mask(t + 1), a.s.qscale, w);
            x = y;
        }
    } else {
        // Half of the waves load K tiles, half V tiles, as in prompt_part: step s puts
        // K of tile s + 1 and V of tile s.
        const int isk = wq < WQ / 2, i0 = wq * LPT - (isk ? 0 : Ge::NL);
        const char *base = uniform_ptr(isk ? a.s.Kt : a.s.Vt);
        unsigned ok = 0;
        u32x4s ld[LPT];
        const auto step = [&](int s, int page) {
#pragma unroll
            for (int j = 0; j < LPT; ++j) load(base, i0 + j, s + isk, page, ld[j], ok, j);
        };
        const auto put = [&](int s) {
            u32x4s *const to = stage + (isk ? ((s + 1) & 1) : 2 + (s & 1)) * Ge::TILE;
#pragma unroll
            for (int j = 0; j < LPT; ++j) {
                if (isk) to[stage_chunk<BF, Ge::S>(Ge::RPI * (i0 + j) + rg, seg)] = ld[j];
                else put_value(ld[j], ((ok >> j) & 1u) && s >= 0, i0 + j, max(s, 0), to);
            }
        };
        // (a step's pages are looked up a step ahead of its loads; step -1 of the V waves has none)
        int pg = pages(max(-1 + isk, 0)), next = pages(isk);
        step(-1, pg);
        load_queries<BF, D, QT>(a.s, it, q0, nq, w);
        lds_barrier();  // (the flags are clear)
        note(0, pg);
        put(-1);
        pg = next, next = pages(1 + isk);
        note(isk, pg);
        step(0, pg);
        put(0);
        pg = next, next = pages(2 + isk);
        note(1 + isk, pg);
        step(1, pg);
        lds_barrier();
        first_tile<BF, D, QT>(stage, x, mask(0), a.s.qscale, w);
        lds_barrier();
        const auto turn = [&](int t, int odd, typename Ge::X &x, typename Ge::X &y) {
            put(t + 1);
            pg = next, next = pages(t + 3 + isk);
            note(t + 2 + isk, pg);
            step(t + 2, pg);
            __builtin_amdgcn_sched_barrier(0);
            if (nq > 0)
                tile_step<BF, D, QT, NS>(stage + (1 - odd) * Ge::TILE, stage + (2 + odd) * Ge::TILE, x, y, mask(t + 1), a.s.qscale, w);
            lds_barrier();
        };
        for (int t = 0; t < tiles; t += 2) {
            turn(t, 0, x, y);
            if (t + 1 >= tiles) break;
            turn(t + 1, 1, y, x);
        }
    }
    if constexpr (WQ == 1) wave_lds_order();
    const unsigned long long bad = flags->bad[0] | (unsigned long long)flags->bad[1] << 32;
    const unsigned long long poison = flags->poison[0] | (unsigned long long)flags->poison[1] << 32;
    if (flags->lost || (bad & sees)) w.ls = NAN;
    write_partials<BF, D, QT>(a.s, it, q0, nq, w);
    if (poison) add_poison<BF, D, QT>(a, it, q0, nq, sees, poison, w.m);
}

template <bool BF, int D, int WQ, int TWQ>
__global__ __launch_bounds__(kShThreads, 2) void k_tree(TreeArgs a)
{
    typedef ShGeo<BF, D, 16> Ge;
    __shared__ u32x4s lds[kShWaves * 2 * Ge::TILE];
    __shared__ TreeFlags flags[kShWaves];
    const uint32_t b = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    const uint32_t prompts = (uint32_t)a.s.grid.prompt_blocks, padded = (prompts + kShXcds - 1) / kShXcds * kShXcds;
    // (each XCD takes a run of the work, in which the tiles of a part are neighbours)
    const auto run = [&](uint32_t b, uint32_t n) {
        const uint32_t x = b % kShXcds;
        return x * (n / kShXcds) + min(x, n % kShXcds) + b / kShXcds;
    };
    if (b < padded) {
        if (b >= prompts) return;
        SharedItem it;
        prompt_item(a.s, run(b, prompts), it);
        if (it.rows > 0) prompt_part<BF, D, WQ, BF ? kTreeSummands : 3>(a.s, it, lds);
    } else {
        const uint32_t tb = b - padded, blocks = (uint32_t)a.tails.blocks;
        if (tb >= blocks) return;
        TreeItem it;
        if constexpr (TWQ == 1) {
            const int wv = uniform_i32(threadIdx.x >> 6);
            const uint32_t w = run(tb, blocks) * kShWaves + wv;
            if (w >= (uint32_t)a.s.grid.tail_waves) return;
            tree_item(a, w, it);
            if (it.rows > 0) tree_part<BF, D, 1>(a, it, lds + wv * 2 * Ge::TILE, flags + wv);
        } else {
            tree_item(a, run(tb, blocks), it);
            if (it.rows > 0) tree_part<BF, D, 4>(a, it, lds, flags);
        }
    }
}

template <bool BF, int D>
static void launch_tree(const TreeArgs &a, dim3 grid, hipStream_t st)
{
    const bool wide = a.s.grid.wq == 4, twide = a.tails.wq == 4;
    if (wide && twide) hipLaunchKernelGGL((k_tree<BF, D, 4, 4>), grid, dim3(kShThreads), 0, st, a);
    else if (wide) hipLaunchKernelGGL((k_tree<BF, D, 4, 1>), grid, dim3(kShThreads), 0, st, a);
    else if (twide) hipLaunchKernelGGL((k_tree<BF, D, 1, 4>), grid, dim3(kShThreads), 0, st, a);
    else hipLaunchKernelGGL((k_tree<BF, D, 1, 1>), grid, dim3(kShThreads), 0, st, a);
}

hipError_t tree_launch(const TreeArgs &a, bool bf16, hipStream_t st)
{
    const int64_t prompts = (a.s.grid.prompt_blocks + kShXcds - 1) / kShXcds * kShXcds;
    const dim3 g = blocks_grid(prompts + a.tails.blocks);
    if (bf16 && a.s.D == 128) ECOKV_TIMED("decode_tree", st, (launch_tree<true, 128>(a, g, st)));
    else if (bf16) ECOKV_TIMED("decode_tree", st, (launch_tree<true, 64>(a, g, st)));
    else if (a.s.D == 128) ECOKV_TIMED("decode_tree", st, (launch_tree<false, 128>(a, g, st)));
    else ECOKV_TIMED("decode_tree", st, (launch_tree<false, 64>(a, g, st)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return merge_launch<true>(a.s, st);
}

}  // namespace ecokv
