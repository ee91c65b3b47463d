// ecokv_decode_tree kernels (gfx950): a tree of drafted tokens of every
// continuation over its prompt's kept rows, its paged tail and the drafted rows
// behind it.
//
// A prompt's kept rows are read by nodes x continuations x G query rows of a
// (layer, KV head), a node in the place of ecokv_decode_shared's continuation: tiles of
// 32 query rows, a wave each (prompt_part), or of 128, whose four waves share the rows
// (wide_part).  A continuation's tail and drafted rows are read by its nodes x G query
// rows: the same tiles, rows found page by page (tree_part).  Node i sees
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

// bf16 summands of a weight in its product with bf16 values.  Two leave out less than
// 2^-14 of it, and what is off in O is then O's own rounding, as for a weight of all its
// bits; one, rounded, would be off by as much again.  Largest error against 64 bits,
// relative, with one, two and three: 0.0023, 0.0017, 0.0017 (with O alone rounded 0.0017).
// (us, the same: 64 nodes on 6553 kept rows of 4 heads 26.6 27.7 30.5; three prompts 34.4
// 36.1 42.6; 64-wide tails of 8000 rows 63.9 64.4 65.8; 28 layers of 4 heads with 6553
// rows, 8 continuations of 130 rows and 16 nodes, bound by matrix work, 445 560 690.)
constexpr int kTreeSummands = 2;

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
    // (parts by the bound, not the count: where a part begins is known before the count is)
    it.row0 = part * a.tails.rows;
    it.rows = valid ? uniform_i32(max(min(n + a.s.nodes - it.row0, a.tails.rows), 0)) : 0;
}

// The b-th of a call's prompt blocks where parts go by the counts (TreeEven): every wave
// takes four units a lane, their steps' sum and the most, and with a part's length the
// blocks of each.  Returns whether there is such a block; `each`: a part's steps.
template <class Run>
__device__ __forceinline__ bool even_item(const TreeArgs &a, uint32_t b, Run run, SharedItem &it, int &each)
{
    constexpr int J = kEvenUnits / kWave;
    const SharedGrid &g = a.s.grid;
    const int lane = threadIdx.x & 63, units = a.s.L * a.s.Hkv * a.s.B;
    const uint32_t step = 2 * (uint32_t)g.rows_t;
    int n[J], off[J], tiles[J], end[J], most = 0;
    float all = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int u = j * kWave + lane;
        n[j] = off[j] = tiles[j] = 0;
        if (j * kWave >= units) continue;
        const int c = a.s.counts[min(u, units - 1)], s = min(u, units - 1) % a.s.B;
        off[j] = a.s.offsets[min(u, units - 1)];
        tiles[j] = g.tile0[s + 1] - g.tile0[s];
        n[j] = u < units && c >= 0 && c <= a.s.max_count ? c : 0;
        const int steps = (int)(((uint32_t)n[j] + step - 1) / step);
        most = max(most, tiles[j] ? steps : 0);
        all += (float)tiles[j] * (float)steps;
    }
    most = (int)wave_max_u32((uint32_t)most);
    all = wave_sum(all);
    const int hi = (most + a.even.least - 1) / a.even.least, lo = (most + g.np - 1) / g.np;
    each = (int)fminf(ceilf(all / (float)a.even.fill), 1e9f);
    each = uniform_i32(max(min(max(each, lo), hi), 1));
    int total = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        end[j] = total;
        if (j * kWave >= units) continue;
        const int steps = (int)(((uint32_t)n[j] + step - 1) / step);
        end[j] += (int)wave_incl_scan((uint32_t)(tiles[j] * ((steps + each - 1) / each)));
        total = __builtin_amdgcn_readlane(end[j], 63);
    }
    if (b >= (uint32_t)total) return false;
    const int w = (int)run(b, (uint32_t)total);
    int u = 0, rows = 0, before = 0;
    bool found = false;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (found || j * kWave >= units) continue;
        const unsigned long long m = __builtin_amdgcn_ballot_w64(end[j] > w);
        if (m) {
            const int i = __ffsll(m) - 1;
            found = true;
            u = j * kWave + i;
            rows = __builtin_amdgcn_readlane(n[j], i);
            it.base = __builtin_amdgcn_readlane(off[j], i);
            const int steps = (int)(((uint32_t)rows + step - 1) / step);
            before = __builtin_amdgcn_readlane(end[j], i) - __builtin_amdgcn_readlane(tiles[j], i) * ((steps + each - 1) / each);
        }
    }
    const int lh = u / a.s.B, s = u - lh * a.s.B, per = g.tile0[s + 1] - g.tile0[s], r = w - before;
    const int part = r / per, tile = r - part * per, qt = g.wq * g.rows_q;
    it.c0 = a.s.fan[s];
    it.nc = a.s.fan[s + 1] - it.c0;
    it.q0 = tile * qt;
    it.nq = min(qt, a.s.G * it.nc - it.q0);
    it.l = lh / a.s.Hkv;
    it.h = lh - it.l * a.s.Hkv;
    it.part = part;
    it.row0 = part * each * (int)step;
    it.rows = min(rows - it.row0, each * (int)step);
    return true;
}

// What lanes of a wave wrote to LDS before is what others read after.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// x of all lanes, joined.
__device__ __forceinline__ uint32_t wave_or_u32(uint32_t x)
{
    x |= dpp_u32<0xB1>(x);
    x |= dpp_u32<0x4E>(x);
    x |= dpp_u32<0x141>(x);
    x |= dpp_u32<0x140>(x);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = (uint32_t)r[0] | (uint32_t)r[1];
    const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (uint32_t)q[0] | (uint32_t)q[1];
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

// The rows of a part for a block's four tiles of query rows, side by side, two tiles of
// rows a step: half of the waves load K, half V, one step ahead in registers and the
// next one in LDS (two places each).  A step is matrix work (logits), vector work
// (weights), matrix work (values): the two blocks of a compute unit put a wave of each on
// every SIMD, and one's matrix work runs beside the other's weights.
//   load(ld, s): the wave's loads of step s;  put(ld, s, ring): into LDS;  mask(t): of
//   tile t's logits.
//   TWICE: the code of a step for each of the two places.
template <bool BF, int D, bool TWICE, class Load, class Put, class Mask>
__device__ __forceinline__ void wide_part(const SharedArgs &a, const SharedItem &it, int q0, int nq, int tiles, Load load, Put put,
                                          Mask mask, u32x4s *stage, ShState<BF, D, BF ? 32 : 16> &w)
{
    constexpr int QT = BF ? 32 : 16;
    typedef ShGeo<BF, D, QT> Ge;
    constexpr int NX = Ge::NX;
    const int lane = threadIdx.x & 63, wq = uniform_i32(threadIdx.x >> 6), grp = lane / QT, row = lane % QT;
    u32x4s *const ring = wq < kShWaves / 2 ? stage : stage + 4 * Ge::TILE;
    u32x4s ld[Ge::NL];
    load(ld, 0);
    load_queries<BF, D, QT>(a, it, q0, nq, w);
    put(ld, 0, ring);
    if (tiles > 2) load(ld, 1);
    const auto step = [&](int t, int odd) __attribute__((always_inline)) {
        const u32x4s *const sk = stage + odd * 2 * Ge::TILE, *const sv = sk + 4 * Ge::TILE;
        // operands are read from LDS AHEAD matrix instructions ahead (the compiler would
        // read each just before its use, a latency of LDS for every pair; 8 ahead left some
        // of the loop's values in scratch memory)
        constexpr int AHEAD = TWICE ? 6 : 4, NV = 4 * Ge::DT;
        bf16x8s op[AHEAD];
        const auto kop = [&](int i) {  // 16 dimensions i / 2 of tile i % 2
            return __builtin_bit_cast(bf16x8s, sk[i % 2 * Ge::TILE + stage_chunk<BF, Ge::S>(row, 2 * (i / 2) + grp)]);
        };
        const auto vop = [&](int i) {  // 16 rows i / DT, tile i % DT of the dimensions
            const int k = i / Ge::DT, r0 = 16 * (k % 2) + 4 * grp;
            return value_operand<Ge::S>(sv + k / 2 * Ge::TILE, r0, r0 + 8, 4 * (i % Ge::DT) + 2 * ((lane >> 4) & 1));
        };
        lds_barrier();
        typename Ge::X x[2];
        if constexpr (BF) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) op[i] = kop(i);
        }
        if (t + 2 < tiles) put(ld, t / 2 + 1, ring + (1 - odd) * 2 * Ge::TILE);
        if (t + 4 < tiles) load(ld, t / 2 + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (nq <= 0) return;
        if constexpr (BF) {
            x[0] = x[1] = (typename Ge::X){};
#pragma unroll
            for (int i = 0; i < 2 * Ge::QS; ++i) {
                x[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i % AHEAD], __builtin_bit_cast(bf16x8s, w.qb[i / 2]), x[i % 2], 0, 0, 0);
                op[i % AHEAD] = i + AHEAD < 2 * Ge::QS ? kop(i + AHEAD) : vop(i + AHEAD - 2 * Ge::QS);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            x[0] = tile_logits<BF, D, QT>(sk, w);
            x[1] = tile_logits<BF, D, QT>(sk + Ge::TILE, w);
        }
        float mb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mb[h] = x[h][0];
#pragma unroll
            for (int r = 1; r < NX; ++r) mb[h] = fmaxf(mb[h], x[h][r]);
            mask(t + h)(x[h], mb[h]);
        }
        tile_reference<BF, D, QT>(fmaxf(mb[0], mb[1]), a.qscale, w);
        const float ref = w.m == -INFINITY ? 0.f : w.m;
        if constexpr (BF) {
            u32x4s p[2][2][kTreeSummands];  // of tile h, rows 16 k ..
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < NX; e += 2) {
                    const float y0 = __builtin_amdgcn_exp2f(fmaf(x[h][e], a.qscale, -ref));
                    const float y1 = __builtin_amdgcn_exp2f(fmaf(x[h][e + 1], a.qscale, -ref));
                    w.ls += y0 + y1;
                    cut_weights(y0, y1, p[h][e / 8], e % 8 / 2);
                }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int k = i / Ge::DT, d = i % Ge::DT, o = (2 * Ge::QS + i) % AHEAD;
#pragma unroll
                for (int j = kTreeSummands - 1; j >= 0; --j)
                    w.acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[o], __builtin_bit_cast(bf16x8s, p[k / 2][k % 2][j]), w.acc[d], 0, 0, 0);
                if (i + AHEAD < NV) op[o] = vop(i + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            tile_values<BF, D, 3>(sv, x[0], a.qscale, w);
            tile_values<BF, D, 3>(sv + Ge::TILE, x[1], a.qscale, w);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (TWICE) {
        for (int t = 0; t < tiles; t += 4) {
            step(t, 0);
            if (t + 2 >= tiles) break;
            step(t + 2, 1);
        }
    } else {
#pragma unroll 1
        for (int t = 0; t < tiles; t += 2) step(t, (t >> 1) & 1);
    }
}

// A block's part of a prompt's unit for its four tiles of query rows.
template <bool BF, int D>
__device__ __forceinline__ void wide_prompt(const SharedArgs &a, const SharedItem &it, u32x4s *stage)
{
    constexpr int QT = BF ? 32 : 16;
    typedef ShGeo<BF, D, QT> Ge;
    const int lane = threadIdx.x & 63, wq = uniform_i32(threadIdx.x >> 6);
    const int q0 = it.q0 + wq * QT, nq = min(it.nq - wq * QT, QT);
    const bool isk = wq < kShWaves / 2;
    const int i0 = (wq & 1) * (Ge::NL / 2);  // the wave's load instructions of a tile
    const int64_t base = (it.base + it.row0) * Ge::RB;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(uniform_ptr((isk ? a.Kc : a.Vc) + base)), (short)0, uniform_i32((int)((uint32_t)it.rows * Ge::RB)), 0x00020000);
    // instruction j: of tile 2 s or the next, rows past the part's read zero
    const auto load = [&](u32x4s (&ld)[Ge::NL], int s) {
#pragma unroll
        for (int j = 0; j < Ge::NL; ++j) {
            const int tile = 2 * s + j / (Ge::NL / 2), i = i0 + j % (Ge::NL / 2);
            ld[j] = __builtin_bit_cast(u32x4s, __builtin_amdgcn_raw_buffer_load_b128(
                rs, (int)((uint32_t)(tile * Ge::TR + Ge::RPI * i) * Ge::RB + lane * 16), 0, 0));
        }
    };
    const auto put = [&](const u32x4s (&ld)[Ge::NL], int, u32x4s *ring) {
#pragma unroll
        for (int j = 0; j < Ge::NL; ++j) {
            const int h = j / (Ge::NL / 2), i = i0 + j % (Ge::NL / 2);
            (ring + h * Ge::TILE)[stage_chunk<BF, Ge::S>(Ge::RPI * i + lane / Ge::S, lane % Ge::S)] = ld[j];
        }
    };
    const auto mask = [&](int t) {
        const int left = it.rows - t * Ge::TR;
        return [left](typename Ge::X &x, float &mb) { tile_mask<BF, D, QT>(x, mb, left, 0u); };
    };
    ShState<BF, D, QT> w;
    wide_part<BF, D, true>(a, it, q0, nq, (it.rows + Ge::TR - 1) / Ge::TR, load, put, mask, stage, w);
    write_partials<BF, D, QT>(a, it, q0, nq, w);
}

// A part of a tail and the drafted rows behind it for one tile of query rows, by
// the four waves of a block (WQ = 4) or by one wave (WQ = 1).
template <bool BF, int D, int WQ>
__device__ __forceinline__ void tree_part(const TreeArgs &a, const TreeItem &it, u32x4s *stage, TreeFlags *flags)
{
    constexpr int QT = BF ? 32 : 16, NS = BF ? kTreeSummands : 3;
    typedef ShGeo<BF, D, QT> Ge;
    constexpr int TR = Ge::TR;
    const int lane = threadIdx.x & 63, wq = WQ == 1 ? 0 : uniform_i32(threadIdx.x >> 6);
    const int seg = lane % Ge::S, rg = lane / Ge::S;
    const int M = a.s.nodes, q0 = it.q0 + wq * QT, nq = min(it.nq - wq * QT, QT);
    const int first = it.n - it.row0;  // of the drafted rows, among the part's
    const bool drafted = first < it.rows;

    // what this lane's node sees of the drafted rows, and what any node does
    const unsigned long long within = M < 64 ? (1ull << M) - 1 : ~0ull;
    unsigned long long sees = 0, any = 0;
    if (drafted) {
        const int m = nq > 0 ? q0 + min(lane % QT, nq - 1) : it.q0;
        sees = a.masks[(int64_t)it.c0 + m % M] & within;
        any = a.masks[(int64_t)it.c0 + min(lane, M - 1)] & within;
    }
    if (WQ == 1 || threadIdx.x == 0) *flags = TreeFlags{};
    if constexpr (WQ == 1) wave_lds_order();

    // the page of this lane's row of a tile (row lane % TR; past 2^31 it is negative), -1 for none
    const auto pages = [&](int t) { return tail_page(a.s.map, it.c, (int)((uint32_t)it.row0 + (uint32_t)(t * TR + lane % TR))); };
    const auto note = [&](int t, int page) {  // rows that have none
        const unsigned lost = (unsigned)__builtin_amdgcn_ballot_w64(page < 0) & (TR == 32 ? ~0u : (1u << (TR & 31)) - 1u);
        if (lost) {
            const int r = t * TR + lane;
            if (page < 0 && lane < TR && r < it.rows) {
                if (r < first) flags->lost = 1;
                else atomicOr(&flags->bad[(r - first) >> 5], 1u << ((r - first) & 31));
            }
        }
        return lost;
    };
    // The n load instructions from i0 on of tile t (rows without a page: of page 0).  A
    // page of at least the rows of an instruction has all of them: one address for the
    // wave, and a lane's place from it never changes.
    const bool whole = (1 << a.s.map.shift) >= Ge::RPI;
    const auto load = [&](const char *base, int i0, int t, int page, auto &x, int at, int n) {
        if (whole) {
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const int pg = __builtin_amdgcn_readlane(page, Ge::RPI * (i0 + j)), row = it.row0 + t * TR + Ge::RPI * (i0 + j);
                const char *p = uniform_ptr(base + tail_row(a.s.map, a.s.Hkv, it.l, it.h, max(pg, 0), row) * Ge::RB);
                x[at + j] = *reinterpret_cast<const u32x4s *>(p + (uint32_t)(lane * 16));
            }
        } else {
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const int pg = __shfl(page, Ge::RPI * (i0 + j) + rg, kWave), row = it.row0 + t * TR + Ge::RPI * (i0 + j) + rg;
                x[at + j] = *reinterpret_cast<const u32x4s *>(
                    base + tail_row(a.s.map, a.s.Hkv, it.l, it.h, max(pg, 0), row) * Ge::RB + 16 * seg);
            }
        }
    };
    // Staged values (instructions i0 .. i0 + n - 1 of tile t, this wave's own) that are not
    // to be read as they are: of rows that nobody sees or that have no page (bits of
    // `lost`), and of drafted rows those that are not finite.  A loop over LDS and not a
    // part of every store: few tiles need it.
    const auto mend_values = [&](int i0, int n, int t, unsigned lost, u32x4s *to) {
        if (t * TR + TR <= min(first, it.rows) && lost == 0) return;
#pragma unroll 1
        for (int i = i0; i < i0 + n; ++i) {
            const int k = Ge::RPI * i + rg, r = t * TR + k;
            u32x4s *const at = to + stage_chunk<BF, Ge::S>(k, seg);
            const bool there = !((lost >> k) & 1) && r < it.rows && (r < first || ((any >> (r - first)) & 1));
            u32x4s x = there ? *at : (u32x4s){0u, 0u, 0u, 0u};
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = odd || not_finite<BF>(x[e]);
            if (odd && r >= first) {
                atomicOr(&flags->poison[(r - first) >> 5], 1u << ((r - first) & 31));
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = finite_part<BF>(x[e]);
            }
            *at = x;
        }
    };
    const auto join = [&]() {  // what any node sees
        if (drafted) any = (unsigned long long)wave_or_u32((uint32_t)(any >> 32)) << 32 | wave_or_u32((uint32_t)any);
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
    if constexpr (WQ == 1) {
        typename Ge::X x, y;
        // K a tile ahead of V, as in prompt_part
        u32x4s kx[Ge::NL], vx[Ge::NL];
        int p1 = pages(1), p2 = pages(2);
        unsigned lost;  // of V's tile
        {
            u32x4s k0[Ge::NL];
            const int p0 = pages(0);
            load(a.s.Kt, 0, 0, p0, k0, 0, Ge::NL);
            load(a.s.Kt, 0, 1, p1, kx, 0, Ge::NL);
            load(a.s.Vt, 0, 0, p0, vx, 0, Ge::NL);
            load_queries<BF, D, QT>(a.s, it, q0, nq, w);
            join();
            lost = note(0, p0);
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) stage[stage_chunk<BF, Ge::S>(Ge::RPI * i + rg, seg)] = k0[i];
        }
        first_tile<BF, D, QT>(stage, x, mask(0), a.s.qscale, w);
        for (int t = 0; t < tiles; ++t) {
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) {
                stage[stage_chunk<BF, Ge::S>(Ge::RPI * i + rg, seg)] = kx[i];
                stage[Ge::TILE + stage_chunk<BF, Ge::S>(Ge::RPI * i + rg, seg)] = vx[i];
            }
            mend_values(0, Ge::NL, t, lost, stage + Ge::TILE);
            lost = note(t + 1, p1);
            load(a.s.Kt, 0, t + 2, p2, kx, 0, Ge::NL);
            load(a.s.Vt, 0, t + 1, p1, vx, 0, Ge::NL);
            p1 = p2;
            p2 = pages(t + 3);
            __builtin_amdgcn_sched_barrier(0);
            tile_step<BF, D, QT, NS>(stage, stage + Ge::TILE, x, y, mask(t + 1), a.s.qscale, w);
            x = y;
        }
    } else {
        const bool isk = wq < WQ / 2;
        const int i0 = (wq & 1) * (Ge::NL / 2);
        const char *base = uniform_ptr(isk ? a.s.Kt : a.s.Vt);
        // pages of a step's two tiles are looked up a step ahead of its loads
        int next[2] = {pages(0), pages(1)};
        unsigned lost[2];
        const auto step = [&](u32x4s (&ld)[Ge::NL], int s) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int pg = next[k];
                next[k] = pages(2 * s + 2 + k);
                load(base, i0, 2 * s + k, pg, ld, k * (Ge::NL / 2), Ge::NL / 2);
                lost[k] = note(2 * s + k, pg);
            }
        };
        const auto put = [&](const u32x4s (&ld)[Ge::NL], int s, u32x4s *ring) {
#pragma unroll
            for (int j = 0; j < Ge::NL; ++j)
                (ring + j / (Ge::NL / 2) * Ge::TILE)[stage_chunk<BF, Ge::S>(Ge::RPI * (i0 + j % (Ge::NL / 2)) + rg, seg)] = ld[j];
            if (isk) return;
            if (s == 0) join();
#pragma unroll 1
            for (int h = 0; h < 2; ++h) mend_values(i0, Ge::NL / 2, 2 * s + h, h ? lost[1] : lost[0], ring + h * Ge::TILE);
        };
        lds_barrier();  // (the flags are clear)
        wide_part<BF, D, false>(a.s, it, q0, nq, tiles, step, put, mask, stage, w);
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
    const uint32_t prompts = (uint32_t)a.s.grid.prompt_blocks, padded = (prompts + kShXcds - 1) / kShXcds * kShXcds;
    const uint32_t blocks = (uint32_t)a.tails.blocks;
    // the prompts' blocks first, or the tails' (TreeEven)
    const uint32_t b0 = blockIdx.z * (uint32_t)kGridX + blockIdx.x, ahead = a.even.ahead ? (blocks + kShXcds - 1) / kShXcds * kShXcds : 0;
    const uint32_t b = b0 - ahead, tb = ahead ? b0 : b0 - padded;  // (past all of the prompts' in the tails' blocks ahead)
    // (each XCD takes a run of the work, in which the tiles of a part are neighbours)
    const auto run = [&](uint32_t b, uint32_t n) {
        const uint32_t x = b % kShXcds;
        return x * (n / kShXcds) + min(x, n % kShXcds) + b / kShXcds;
    };
    if (b < padded) {
        if (b >= prompts) return;
        SharedItem it;
        if (WQ == 4 && a.even.fill > 0) {
            int each;
            const bool there = even_item(a, b, run, it, each);
            if (b == 0 && threadIdx.x == 0) a.s.part_steps[0] = each;
            if (!there) return;
        } else {
            prompt_item(a.s, run(b, prompts), it);
        }
        if (it.rows > 0) {
            if constexpr (WQ == 1) prompt_part<BF, D, 1, BF ? kTreeSummands : 3>(a.s, it, lds);
            else wide_prompt<BF, D>(a.s, it, lds);
        }
    } else {
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
    const bool wide = a.s.grid.wq == 4;
    if (a.tails.wq == 4) {
        if (wide) hipLaunchKernelGGL((k_tree<BF, D, 4, 4>), grid, dim3(kShThreads), 0, st, a);
        else hipLaunchKernelGGL((k_tree<BF, D, 1, 4>), grid, dim3(kShThreads), 0, st, a);
    } else if constexpr (!(BF && D == 128)) {
        if (wide) hipLaunchKernelGGL((k_tree<BF, D, 4, 1>), grid, dim3(kShThreads), 0, st, a);
        else hipLaunchKernelGGL((k_tree<BF, D, 1, 1>), grid, dim3(kShThreads), 0, st, a);
    }
}

hipError_t tree_launch(const TreeArgs &a, bool bf16, hipStream_t st)
{
    const int64_t prompts = (a.s.grid.prompt_blocks + kShXcds - 1) / kShXcds * kShXcds;
    const dim3 g = blocks_grid(prompts + (a.tails.blocks + kShXcds - 1) / kShXcds * kShXcds);
    if (bf16 && a.s.D == 128) ECOKV_TIMED("decode_tree", st, (launch_tree<true, 128>(a, g, st)));
    else if (bf16) ECOKV_TIMED("decode_tree", st, (launch_tree<true, 64>(a, g, st)));
    else if (a.s.D == 128) ECOKV_TIMED("decode_tree", st, (launch_tree<false, 128>(a, g, st)));
    else ECOKV_TIMED("decode_tree", st, (launch_tree<false, 64>(a, g, st)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return merge_launch<true>(a.s, st);
}

}  // namespace ecokv
