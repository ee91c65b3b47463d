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
#include <type_traits>

#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4s __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8s __attribute__((ext_vector_type(8)));
typedef float f32x4s __attribute__((ext_vector_type(4)));
typedef float f32x16s __attribute__((ext_vector_type(16)));
typedef short s16x4s __attribute__((ext_vector_type(4)));

constexpr int kShThreads = kShWaves * kWave;
constexpr uint32_t kShXcds = 8;   // XCDs, to which blocks are dealt in turn
constexpr float kShRebase = 8.f;  // log2 headroom of the lazily moved reference

// Work of a block (or, in the tails, of a wave): query rows q0 .. q0 + nq - 1 of
// the nc continuations from c0 on (row m: head m / nc of the group, continuation
// c0 + m % nc), rows [row0, row0 + rows) of the prompt's unit or of the tail of
// continuation c0, and the part of the workspace that takes the partials.
struct SharedItem {
    int l, h, c0, nc, q0, nq, row0, rows, part;
    int64_t base;  // first row of the prompt's unit
};

__device__ __forceinline__ void item_rows(SharedItem &it, int n, int most, int parts, int part, int step)
{
    n = n < 0 || n > most ? 0 : n;  // (counts out of their bounds: the merge writes NaN)
    const uint32_t pr = part_rows(n, parts, step);
    const uint64_t r0 = (uint64_t)(uint32_t)part * pr;
    it.row0 = uniform_i32((int)min(r0, (uint64_t)n));
    it.rows = uniform_i32((int)min((uint32_t)(n - it.row0), pr));
}

__device__ __forceinline__ void prompt_item(const SharedArgs &a, uint32_t b, SharedItem &it)
{
    const SharedGrid &g = a.grid;
    const uint32_t per = (uint32_t)(g.tiles * g.np);
    const int qt = g.wq * g.rows_q;
    const int lh = (int)(b / per), r = (int)(b - (uint32_t)lh * per);
    const int part = (int)((uint32_t)r / (uint32_t)g.tiles), tile = r - part * g.tiles;
    int s = 0;
    while (s + 1 < a.B && g.tile0[s + 1] <= tile) ++s;
    const int64_t u = (int64_t)lh * a.B + s;
    const int n = uniform_i32(a.counts[u]), off = uniform_i32(a.offsets[u]);
    it.c0 = a.fan[s];
    it.nc = a.fan[s + 1] - it.c0;
    it.q0 = (tile - g.tile0[s]) * qt;
    it.nq = min(qt, a.G * it.nc - it.q0);
    it.l = (int)((uint32_t)lh / (uint32_t)a.Hkv);
    it.h = lh - it.l * a.Hkv;
    it.part = part;
    it.base = off;
    item_rows(it, n, a.max_count, g.np, part, g.step);
}

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

// Shapes of a wave's work: QT query rows (bf16 32 or 16, fp32 16) and a tile of
// the cache's rows.
template <bool BF, int D, int QT>
struct ShGeo {
    static constexpr int TR = BF ? 32 : 16;       // rows of a tile
    static constexpr int RB = D * (BF ? 2 : 4);   // row bytes
    static constexpr int S = RB / 16;             // 16-byte chunks per row
    static constexpr int RPI = kWave / S;         // rows per load instruction
    static constexpr int NL = TR / RPI;           // load instructions for K, and for V
    static constexpr int GR = kWave / QT;         // lane groups, each with its own rows and dimensions
    static constexpr int QS = S / GR;             // 16-byte operands of a query row per lane
    static constexpr int NX = TR / GR;            // logits per lane
    static constexpr int DT = D / QT;             // tiles of the output's dimensions
    static constexpr int AX = QT / GR;            // sums of a tile per lane
    static constexpr int TILE = TR * S;           // chunks of K (or V) of a tile
    typedef float X __attribute__((ext_vector_type(NX)));
    typedef float A __attribute__((ext_vector_type(AX)));
};

// Place of chunk c of row r of a staged tile.  Row-wise writes, the K operand
// (16 rows' chunk c) and the V operand (bf16: 4 adjacent rows' 64 bytes per
// half-wave; fp32: 64 bytes of rows 4 apart) each spread over all banks.
template <bool BF, int S>
__device__ __forceinline__ int stage_chunk(int r, int c)
{
    if constexpr (!BF) return r * S + (c ^ (r & 15));
    else if constexpr (S == 16) return r * S + (c ^ (((r & 3) << 2) | ((r >> 2) & 3)));
    else return r * S + (c ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3)));
}

// A wave's state: its query row's reference maximum (base 2), sum (this lane's
// part of it) and weighted values.
template <bool BF, int D, int QT>
struct ShState {
    u32x4s qb[ShGeo<BF, D, QT>::QS];
    typename ShGeo<BF, D, QT>::A acc[ShGeo<BF, D, QT>::DT];
    float m, ls;
};

// Query rows q0 .. q0 + nq - 1 of the item as operand B (rows past nq repeat the
// last; none at all: the first of the item).
template <bool BF, int D, int QT>
__device__ __forceinline__ void load_queries(const SharedArgs &a, const SharedItem &it, int q0, int nq, ShState<BF, D, QT> &w)
{
    typedef ShGeo<BF, D, QT> Ge;
    const int lane = threadIdx.x & 63;
    const int m = nq > 0 ? q0 + min(lane % QT, nq - 1) : it.q0, g = m / it.nc, c = it.c0 + m % it.nc;
    const char *q = a.Q + (((int64_t)it.l * a.Hq + it.h * a.G + g) * a.N + c) * Ge::RB + 16 * (lane / QT);
#pragma unroll
    for (int st = 0; st < Ge::QS; ++st) w.qb[st] = *reinterpret_cast<const u32x4s *>(q + 16 * Ge::GR * st);
    w.m = -INFINITY;
    w.ls = 0.f;
#pragma unroll
    for (int d = 0; d < Ge::DT; ++d) w.acc[d] = (typename Ge::A){};
}

// Row of a tile that logit r of a lane belongs to.
template <bool BF, int D, int QT>
__device__ __forceinline__ int tile_key(int r)
{
    const int grp = (threadIdx.x & 63) / QT;
    return QT == 32 ? 8 * (r >> 2) + 4 * grp + (r & 3) : 16 * (r >> 2) + 4 * grp + (r & 3);
}

// Logits (unscaled) of a staged tile's rows against the wave's query rows.
template <bool BF, int D, int QT>
__device__ __forceinline__ typename ShGeo<BF, D, QT>::X tile_logits(const u32x4s *sk, const ShState<BF, D, QT> &w)
{
    typedef ShGeo<BF, D, QT> Ge;
    const int lane = threadIdx.x & 63, grp = lane / QT, row = lane % QT;
    const auto chunk = [&](int t, int s) { return sk[stage_chunk<BF, Ge::S>(QT * t + row, Ge::GR * s + grp)]; };
    typename Ge::X x = (typename Ge::X){};
    if constexpr (QT == 32) {
#pragma unroll
        for (int s = 0; s < Ge::QS; ++s)
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8s, chunk(0, s)),
                                                        __builtin_bit_cast(bf16x8s, w.qb[s]), x, 0, 0, 0);
    } else if constexpr (BF) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4s y = {};
#pragma unroll
            for (int s = 0; s < Ge::QS; ++s)
                y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8s, chunk(t, s)),
                                                            __builtin_bit_cast(bf16x8s, w.qb[s]), y, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * t + r] = y[r];
        }
    } else {
        // (four chains: a quarter of the latency and of the roundings in a row)
        f32x4s y[4] = {};
#pragma unroll
        for (int s = 0; s < Ge::QS; ++s) {
            const u32x4s k = chunk(0, s);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(w.qb[s][e]), y[e], 0, 0, 0);
        }
        x = (y[0] + y[1]) + (y[2] + y[3]);
    }
    return x;
}

// Masks a tile's logits, whose largest is mb: `left` of its rows exist; rows of
// `bad` have no page and give NaN.
template <bool BF, int D, int QT>
__device__ __forceinline__ void tile_mask(typename ShGeo<BF, D, QT>::X &x, float &mb, int left, unsigned bad)
{
    typedef ShGeo<BF, D, QT> Ge;
    if (left < Ge::TR || bad) {
        __builtin_amdgcn_sched_barrier(0);  // (a branch: as selects it would cost a fifth of a tile's vector work)
        mb = -INFINITY;
#pragma unroll
        for (int r = 0; r < Ge::NX; ++r) {
            const int k = tile_key<BF, D, QT>(r);
            if ((bad >> k) & 1u) x[r] = NAN;
            if (k >= left) x[r] = -INFINITY;
            mb = fmaxf(mb, x[r]);
        }
    }
}

// Moves the reference where a tile's largest logit mb (of this lane's rows) needs it.
template <bool BF, int D, int QT>
__device__ __forceinline__ void tile_reference(float mb, float qscale, ShState<BF, D, QT> &w)
{
    typedef ShGeo<BF, D, QT> Ge;
    if constexpr (QT == 16) mb = across16(mb, OpMax{});
    mb = across32(mb, OpMax{}) * qscale;
    const bool move = mb > w.m + kShRebase;  // (from m = -inf: with the first finite logit)
    if (__builtin_amdgcn_ballot_w64(move)) {
        const float nm = move ? mb : w.m;
        const float sc = move ? __builtin_amdgcn_exp2f(w.m - nm) : 1.f;  // 0 while m = -inf
        w.m = nm;
        w.ls *= sc;
#pragma unroll
        for (int d = 0; d < Ge::DT; ++d)
#pragma unroll
            for (int r = 0; r < Ge::AX; ++r) w.acc[d][r] *= sc;
    }
}

// The first tile's logits, and the reference for them.
template <bool BF, int D, int QT>
__device__ __forceinline__ void first_tile(const u32x4s *sk, typename ShGeo<BF, D, QT>::X &x, int left, unsigned bad, float qscale,
                                           ShState<BF, D, QT> &w)
{
    x = tile_logits<BF, D, QT>(sk, w);
    float mb = x[0];
#pragma unroll
    for (int r = 1; r < ShGeo<BF, D, QT>::NX; ++r) mb = fmaxf(mb, x[r]);
    tile_mask<BF, D, QT>(x, mb, left, bad);
    tile_reference<BF, D, QT>(mb, qscale, w);
}

// The weights y0, y1 of two rows as dword j of the three summands p.  Cut, not
// rounded: what is left is exact, and the third summand the rest.  (The bf16 dot
// instruction would take a fifth fewer, but not beside a matrix one.)
__device__ __forceinline__ void cut_weights(float y0, float y1, u32x4s (&p)[3], int j)
{
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        p[k][j] = __builtin_amdgcn_perm(__float_as_uint(y1), __float_as_uint(y0), 0x07060302u);
        if (k < 2) {
            y0 -= __uint_as_float(__float_as_uint(y0) & 0xffff0000u);
            y1 -= __uint_as_float(__float_as_uint(y1) & 0xffff0000u);
        }
    }
}

// Operand of V^T: two times four rows row0 + 4 grp .. and row1 + 4 grp .. of a
// staged tile, dimensions dim0 .. (16 of them per 16 lanes).
template <int S>
__device__ __forceinline__ bf16x8s value_operand(const u32x4s *sv, int row0, int row1, int chunk0)
{
    const uint16_t *sv16 = reinterpret_cast<const uint16_t *>(sv);
    const int i = threadIdx.x & 15, c = chunk0 + ((i & 3) >> 1), off = (i & 1) * 4;
    s16x4s v[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
        v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4s *)(
            const_cast<uint16_t *>(sv16 + 8 * stage_chunk<true, S>((t ? row1 : row0) + (i >> 2), c) + off)));
    const short __attribute__((ext_vector_type(8))) v8 = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
    return __builtin_bit_cast(bf16x8s, v8);
}

// A tile's values (staged at sv) added up with the weights of its logits x, in
// their order: 16 query rows (the tails, and fp32).
template <bool BF, int D>
__device__ __forceinline__ void tile_values(const u32x4s *sv, const typename ShGeo<BF, D, 16>::X &x, float qscale, ShState<BF, D, 16> &w)
{
    typedef ShGeo<BF, D, 16> Ge;
    const int lane = threadIdx.x & 63, grp = lane >> 4, row = lane & 15;
    const float ref = w.m == -INFINITY ? 0.f : w.m;
    float p[Ge::NX];
#pragma unroll
    for (int r = 0; r < Ge::NX; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(x[r], qscale, -ref));
        w.ls += p[r];
    }
    if constexpr (BF) {
        u32x4s c[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) cut_weights(p[2 * j], p[2 * j + 1], c, j);
#pragma unroll
        for (int d = 0; d < Ge::DT; ++d) {
            const bf16x8s v = value_operand<Ge::S>(sv, 4 * grp, 16 + 4 * grp, 2 * d);
#pragma unroll
            for (int k = 2; k >= 0; --k)
                w.acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8s, c[k]), w.acc[d], 0, 0, 0);
        }
    } else {
        const float *sv32 = reinterpret_cast<const float *>(sv);
#pragma unroll
        for (int d = 0; d < Ge::DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = sv32[4 * stage_chunk<BF, Ge::S>(4 * grp + r, 4 * d + (row >> 2)) + (row & 3)];
                w.acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[r], w.acc[d], 0, 0, 0);
            }
    }
}

// A tile's values (staged at sv) added up with the weights of its logits x, and
// the next tile's logits y (K staged at sk; `left` and `bad` as tile_mask) with
// the reference for them.  32 query rows: a matrix instruction takes the time of
// six or seven vector ones, which run beside it if they stand there: the two
// matrix instructions of a pair of the next logits beside the first half's
// weights, the first half's values beside the second half's weights, the second
// half's beside the next logits' maximum; and operands are read from LDS ahead.
template <bool BF, int D, int QT>
__device__ __forceinline__ void tile_step(const u32x4s *sk, const u32x4s *sv, const typename ShGeo<BF, D, QT>::X &x,
                                          typename ShGeo<BF, D, QT>::X &y, int left, float qscale, ShState<BF, D, QT> &w)
{
    typedef ShGeo<BF, D, QT> Ge;
    constexpr int S = Ge::S, NX = Ge::NX;
    float mb = -INFINITY;
    if constexpr (QT == 32) {
        const int lane = threadIdx.x & 63, grp = lane >> 5, row = lane & 31;
        const float ref = w.m == -INFINITY ? 0.f : w.m;
        const auto kop = [&](int s) { return __builtin_bit_cast(bf16x8s, sk[stage_chunk<BF, S>(row, 2 * s + grp)]); };
        // 16 rows g / DT, dimensions 32 (g % DT) ..
        const auto vop = [&](int g) {
            const int r0 = 16 * (g / Ge::DT) + 4 * grp;
            return value_operand<S>(sv, r0, r0 + 8, 4 * (g % Ge::DT) + 2 * ((lane >> 4) & 1));
        };
        u32x4s p[2][3];
        const auto weights = [&](int e) {  // of rows e, e + 1
            const float y0 = __builtin_amdgcn_exp2f(fmaf(x[e], qscale, -ref)), y1 = __builtin_amdgcn_exp2f(fmaf(x[e + 1], qscale, -ref));
            w.ls += y0 + y1;
            cut_weights(y0, y1, p[e / 8], e % 8 / 2);
        };
        constexpr int G = 2 * Ge::DT;  // value operands
        bf16x8s kf[2] = {kop(0), kop(1)}, vf[2];
        y = (typename Ge::X){};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < Ge::QS; ++s) {
            y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s & 1], __builtin_bit_cast(bf16x8s, w.qb[s]), y, 0, 0, 0);
            if (s + 2 < Ge::QS) kf[s & 1] = kop(s + 2);
            if (s & 1) {
                if (s + 1 == Ge::QS) vf[0] = vop(0);
#pragma unroll
                for (int e = 0; e < 16 / Ge::QS; e += 2) weights((s / 2) * (16 / Ge::QS) + e);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int d = g % Ge::DT;
            if (g + 1 < G) vf[(g + 1) & 1] = vop(g + 1);
#pragma unroll
            for (int k = 2; k >= 0; --k)
                w.acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[g & 1], __builtin_bit_cast(bf16x8s, p[g / Ge::DT][k]), w.acc[d], 0, 0, 0);
            if (g < Ge::DT) {
#pragma unroll
                for (int e = 0; e < 8 / Ge::DT; e += 2) weights(8 + d * (8 / Ge::DT) + e);
            } else {
#pragma unroll
                for (int r = 0; r < NX / Ge::DT; ++r) mb = fmaxf(mb, y[d * (NX / Ge::DT) + r]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        y = tile_logits<BF, D, QT>(sk, w);
#pragma unroll
        for (int r = 0; r < NX; ++r) mb = fmaxf(mb, y[r]);
        tile_values<BF, D>(sv, x, qscale, w);
    }
    tile_mask<BF, D, QT>(y, mb, left, 0u);
    tile_reference<BF, D, QT>(mb, qscale, w);
}

// Dimension of the first of four consecutive sums 4 r4 .. of tile d.
template <int QT>
__device__ __forceinline__ int sum_dim(int d, int r4)
{
    return QT * d + 8 * r4 + 4 * ((threadIdx.x & 63) / QT);
}

// Place of query row m of an item in a part of the workspace.
__device__ __forceinline__ int64_t partial_row(const SharedArgs &a, const SharedItem &it, int m)
{
    return (int64_t)it.part * a.grid.qrows + ((int64_t)it.l * a.Hq + it.h * a.G + m / it.nc) * a.N + it.c0 + m % it.nc;
}

template <int QT>
__device__ __forceinline__ float sum_groups(float v)
{
    if constexpr (QT == 16) v = across16(v, OpAdd{});
    return across32(v, OpAdd{});
}

// A wave's partials straight from its registers.
template <bool BF, int D, int QT>
__device__ __forceinline__ void write_partials(const SharedArgs &a, const SharedItem &it, int q0, int nq, const ShState<BF, D, QT> &w)
{
    typedef ShGeo<BF, D, QT> Ge;
    const int lane = threadIdx.x & 63, q = lane % QT;
    const float ls = sum_groups<QT>(w.ls);
    if (q >= nq) return;
    const int64_t row = partial_row(a, it, q0 + q);
#pragma unroll
    for (int d = 0; d < Ge::DT; ++d)
#pragma unroll
        for (int r4 = 0; r4 < Ge::AX / 4; ++r4)
            *reinterpret_cast<f32x4s *>(a.acc + row * D + sum_dim<QT>(d, r4)) =
                (f32x4s){w.acc[d][4 * r4], w.acc[d][4 * r4 + 1], w.acc[d][4 * r4 + 2], w.acc[d][4 * r4 + 3]};
    if (lane < QT) a.ms[row] = make_float2(w.m, ls);
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
        first_tile<BF, D, 16>(stage, x, left, bad, a.qscale, w);
        tile_values<BF, D>(stage + Ge::TILE, x, a.qscale, w);
    }
    write_partials<BF, D, 16>(a, it, it.q0, it.nq, w);
}

// A block's part of a prompt's unit.  4 / WQ groups of WQ waves: a group's waves
// load its tiles together, each for its own query rows.
template <bool BF, int D, int WQ>
__device__ __forceinline__ void prompt_part(const SharedArgs &a, const SharedItem &it, u32x4s *lds)
{
    constexpr int QT = BF ? 32 : 16;
    typedef ShGeo<BF, D, QT> Ge;
    constexpr int KG = kShWaves / WQ, LPT = 2 * Ge::NL / WQ;  // groups; load instructions of a wave for a tile
    const int lane = threadIdx.x & 63, wv = uniform_i32(threadIdx.x >> 6);
    const int kgi = wv / WQ, wq = wv % WQ;
    const int share = (it.rows + KG - 1) / KG;
    const int per = (share + Ge::TR - 1) / Ge::TR * Ge::TR;  // rows of a group
    const int first = min(kgi * per, it.rows), nrows = min(it.rows - first, per);
    const int tiles = per / Ge::TR;                          // (of every group, for the barriers)
    const int q0 = it.q0 + wq * QT, nq = min(it.nq - wq * QT, QT);
    const int64_t base = (it.base + it.row0 + first) * Ge::RB;
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(uniform_ptr(a.Kc + base)), (short)0, uniform_i32((int)((uint32_t)nrows * Ge::RB)), 0x00020000);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(uniform_ptr(a.Vc + base)), (short)0, uniform_i32((int)((uint32_t)nrows * Ge::RB)), 0x00020000);
    u32x4s *const stage = lds + kgi * (WQ > 1 ? 4 : 2) * Ge::TILE;
    ShState<BF, D, QT> w;
    if constexpr (WQ == 1) {
        // each wave its own tiles, a step ahead in registers (rows past the wave's
        // read zero); K a tile ahead of V, as below
        u32x4s kx[Ge::NL], vx[Ge::NL];
        const auto load = [&](u32x4s (&x)[Ge::NL], __amdgpu_buffer_rsrc_t rs, int t) {
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i)
                x[i] = __builtin_bit_cast(u32x4s, __builtin_amdgcn_raw_buffer_load_b128(
                    rs, (int)((uint32_t)(t * Ge::TR + Ge::RPI * i) * Ge::RB + lane * 16), 0, 0));
        };
        const auto put = [&](const u32x4s (&x)[Ge::NL], u32x4s *to) {
#pragma unroll
            for (int i = 0; i < Ge::NL; ++i) to[stage_chunk<BF, Ge::S>(Ge::RPI * i + lane / Ge::S, lane % Ge::S)] = x[i];
        };
        {  // (the first tiles' loads together: one round trip)
            u32x4s k0[Ge::NL];
            load(k0, rk, 0);
            load(kx, rk, 1);
            load(vx, rv, 0);
            load_queries<BF, D, QT>(a, it, q0, nq, w);
            put(k0, stage);
        }
        typename Ge::X x, y;
        first_tile<BF, D, QT>(stage, x, nrows, 0u, a.qscale, w);
        for (int t = 0; t * Ge::TR < nrows; ++t) {
            put(kx, stage);
            put(vx, stage + Ge::TILE);
            load(kx, rk, t + 2);
            load(vx, rv, t + 1);
            __builtin_amdgcn_sched_barrier(0);
            tile_step<BF, D, QT>(stage, stage + Ge::TILE, x, y, nrows - (t + 1) * Ge::TR, a.qscale, w);
            x = y;
        }
    } else {
        // Half of a group's waves load K tiles, half V tiles, one ahead in
        // registers and the next one in LDS.  K runs a tile ahead of V: the next
        // tile's logits are matrix work that fills the softmax of this one.  Step
        // s puts K of tile s + 1 and V of tile s (V of tile -1: zeros).
        const bool isk = wq < WQ / 2;
        const int i0 = wq * LPT - (isk ? 0 : Ge::NL);  // first of the wave's load instructions
        const __amdgpu_buffer_rsrc_t rs = isk ? rk : rv;
        const auto load = [&](u32x4s (&ld)[LPT], int s) {
#pragma unroll
            for (int j = 0; j < LPT; ++j)
                ld[j] = __builtin_bit_cast(u32x4s, __builtin_amdgcn_raw_buffer_load_b128(
                    rs, (int)((uint32_t)((s + (isk ? 1 : 0)) * Ge::TR + Ge::RPI * (i0 + j)) * Ge::RB + lane * 16), 0, 0));
        };
        // K tiles at stage + (tile & 1) TILE, V tiles two TILEs on
        const auto put = [&](const u32x4s (&ld)[LPT], int s) {
            u32x4s *const to = stage + (isk ? ((s + 1) & 1) : 2 + (s & 1)) * Ge::TILE;
#pragma unroll
            for (int j = 0; j < LPT; ++j)
                to[stage_chunk<BF, Ge::S>(Ge::RPI * (i0 + j) + lane / Ge::S, lane % Ge::S)] = ld[j];
        };
        u32x4s ld[LPT];
        {  // (the first steps' loads together: one round trip)
            u32x4s l0[LPT];
            load(ld, -1);
            load(l0, 0);
            load_queries<BF, D, QT>(a, it, q0, nq, w);
            put(ld, -1);
            load(ld, 1);
            put(l0, 0);
        }
        lds_barrier();
        typename Ge::X x, y;
        first_tile<BF, D, QT>(stage, x, nrows, 0u, a.qscale, w);
        lds_barrier();  // (the first turn puts tile 2 in its place)
        // tile t, even or odd: its V, the next tile's K, and the step after both
        const auto turn = [&](int t, int odd, typename Ge::X &x, typename Ge::X &y) {
            put(ld, t + 1);
            load(ld, t + 2);
            __builtin_amdgcn_sched_barrier(0);
            if (nq > 0)
                tile_step<BF, D, QT>(stage + (1 - odd) * Ge::TILE, stage + (2 + odd) * Ge::TILE, x, y, nrows - (t + 1) * Ge::TR,
                                     a.qscale, w);
            lds_barrier();
        };
        for (int t = 0; t < tiles; t += 2) {
            turn(t, 0, x, y);
            if (t + 1 >= tiles) break;
            turn(t + 1, 1, y, x);
        }
    }
    if constexpr (KG == 1) {
        write_partials<BF, D, QT>(a, it, q0, nq, w);
    } else {
        // The groups' waves of the same query rows join their partials: each scales its
        // sums to the common reference and finishes 1 / KG of them, the others' shares
        // through LDS.  (Sums in query-row order in LDS, joined by all threads with a
        // division for each one's place, took 3 us longer: eight continuations of
        // 6553 rows 20.1 -> 18.5.)
        __shared__ float wm[kShWaves][QT], wl[kShWaves][QT];
        constexpr int C4 = Ge::AX / 4, C = Ge::DT * C4, OWN = C / KG;  // chunks of four sums of a lane
        const float ls = sum_groups<QT>(w.ls);
        const int q = lane % QT;
        if (lane < QT) {
            wm[wv][q] = w.m;
            wl[wv][q] = ls;
        }
        __syncthreads();  // (every stage has been read, too)
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int k = 0; k < KG; ++k) M = fmaxf(M, wm[k * WQ + wq][q]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int k = 0; k < KG; ++k) L += wl[k * WQ + wq][q] * __builtin_amdgcn_exp2f(wm[k * WQ + wq][q] - ref);
        const float mine = __builtin_amdgcn_exp2f(w.m - ref);
        f32x4s *const shares = reinterpret_cast<f32x4s *>(lds);  // [wave][chunk][lane]
        f32x4s own[OWN];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const f32x4s v = (f32x4s){w.acc[c / C4][4 * (c % C4)], w.acc[c / C4][4 * (c % C4) + 1], w.acc[c / C4][4 * (c % C4) + 2],
                                      w.acc[c / C4][4 * (c % C4) + 3]} * mine;
            if (c / OWN != kgi) shares[(wv * C + c) * kWave + lane] = v;
            else own[c % OWN] = v;
        }
        __syncthreads();
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const int from = (kgi + k) % KG * WQ + wq;
#pragma unroll
            for (int c = 0; c < OWN; ++c) own[c] += shares[(from * C + kgi * OWN + c) * kWave + lane];
        }
        if (q >= nq) return;
        const int64_t row = partial_row(a, it, q0 + q);
#pragma unroll
        for (int c = 0; c < OWN; ++c) {
            const int cc = kgi * OWN + c;
            *reinterpret_cast<f32x4s *>(a.acc + row * D + sum_dim<QT>(cc / C4, cc % C4)) = own[c];
        }
        if (kgi == 0 && lane < QT) a.ms[row] = make_float2(M, L);
    }
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
        if (it.rows > 0) prompt_part<BF, D, WQ>(a, it, lds);
    } else {
        const int wv = uniform_i32(threadIdx.x >> 6);
        const uint32_t w = (b - prompts) * kShWaves + wv;
        if (w >= (uint32_t)a.grid.tail_waves) return;
        tail_item(a, w, it);
        if (it.rows > 0) tail_part<BF, D>(a, it, lds + wv * 2 * Ge::TILE);
    }
}

// The partials of a query row: np prompt parts and nt tail parts of those that
// the workspace has places for, none (and NaN outputs) where a count is out of
// its bounds.
struct ShParts {
    int np, nt;
    bool bad;
};
__device__ __forceinline__ ShParts row_parts(const SharedArgs &a, uint32_t qrow)
{
    const uint32_t lq = qrow / (uint32_t)a.N, lh = lq / (uint32_t)a.G;  // (heads of a group are neighbours in every layer)
    const int c = (int)(qrow - lq * (uint32_t)a.N);
    ShParts r{0, 0, false};
    if (a.max_count > 0) {
        int s = 0;
        while (s + 1 < a.B && a.fan[s + 1] <= c) ++s;
        const int n = a.counts[(int64_t)lh * a.B + s];
        r.bad = n < 0 || n > a.max_count;
        r.np = r.bad ? 0 : parts_used(n, a.grid.np, a.grid.step);
    }
    if (a.max_tail > 0) {
        const int n = a.tail_counts[c];
        r.bad = r.bad || n < 0 || n > a.max_tail;
        r.nt = n < 0 || n > a.max_tail ? 0 : parts_used(n, a.grid.nt, a.grid.tail_step);
    }
    return r;
}
// Whether place k of the workspace holds one of them.
__device__ __forceinline__ bool has_part(const SharedArgs &a, const ShParts &r, int k)
{
    return k < a.grid.np ? k < r.np : k - a.grid.np < r.nt;
}

// O and lse of a query row from its merged (reference, sum) and four sums.
__device__ __forceinline__ void write_out(const SharedArgs &a, uint32_t qrow, int d, bool bad, float M, float L, f32x4s o)
{
    // (L is 0 without rows and where every logit is -inf, NaN where one is)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = bad ? NAN : (L == 0.f ? 0.f : o[e] / L);
    *reinterpret_cast<f32x4s *>(a.O + (int64_t)qrow * a.D + d) = o;
    if (d == 0 && a.lse) a.lse[qrow] = bad ? NAN : (L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f);
}

// Up to kShFew partials: D / 4 threads per query row, every place of the
// workspace loaded at once, ahead of the counts that say which hold a partial
// (the others' contents are not used).  A call without kept rows and tails has
// no places.
// The forms load FEW places whatever a call has, so a call takes the next one up,
// and past the last k_shared_merge.  us a merge out of a graph, D = 128, forms of
// 2, 3, 5, 8, 14, 24 places and a block a row: 1792 query rows, 2 partials 2.6 2.7
// 2.9 3.1 3.6 4.5 5.7, 5 partials - - 3.2 3.4 4.0 4.8 6.1, 12 - - - - 4.8 5.7 6.2,
// 20 - - - - - 6.6 6.2, 24 7.0 and 6.2; 12544 rows, 2 partials 4.6 4.9 5.5 6.5 9.0
// 15.9 22.8, 5 - - 7.2 8.0 10.6 18.3 25.7, 12 - - - - 16.1 25.3 26.6, 24 34 and 28
// (D = 64: 21 and 28).  The rule does not look at the rows: with few of them a block
// a row is as fast from 6 to 8 partials on (224 rows: 6 partials 3.4 3.5, 12 4.7 3.5, 20
// 6.4 3.5).
constexpr int kShMergeThreads = 256, kShFew = 24;
template <int D, int FEW>
__global__ __launch_bounds__(kShMergeThreads) void k_shared_merge_few(SharedArgs a)
{
    constexpr int ROWS = kShMergeThreads / (D / 4);
    const uint32_t qrow = (blockIdx.z * (uint32_t)kGridX + blockIdx.x) * ROWS + threadIdx.x / (D / 4);
    if (qrow >= (uint32_t)a.grid.qrows) return;
    const int d = 4 * (threadIdx.x % (D / 4)), P = a.grid.np + a.grid.nt;
    if (P == 0) {
        write_out(a, qrow, d, false, -INFINITY, 0.f, (f32x4s){});
        return;
    }
    f32x4s v[FEW];
    float2 e[FEW];
#pragma unroll
    for (int k = 0; k < FEW; ++k) {
        const int64_t row = (int64_t)min(k, P - 1) * a.grid.qrows + qrow;
        e[k] = a.ms[row];
        v[k] = *reinterpret_cast<const f32x4s *>(a.acc + row * D + d);
    }
    const ShParts r = row_parts(a, qrow);
    float M = -INFINITY, L = 0.f;
    f32x4s o = {};
#pragma unroll
    for (int k = 0; k < FEW; ++k)
        if (k < P && has_part(a, r, k)) M = fmaxf(M, e[k].x);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int k = 0; k < FEW; ++k)
        if (k < P && has_part(a, r, k)) {
            const float w = exp2f(e[k].x - ref);
            L += e[k].y * w;
            o += v[k] * w;
        }
    write_out(a, qrow, d, r.bad, M, L, o);
}

// One block per query row: thread t weighs partial t, 256 at a time; groups of
// D / 4 threads add up the sums, each every (1024 / D)-th.
template <int D>
__global__ __launch_bounds__(kShMergeThreads) void k_shared_merge(SharedArgs a)
{
    constexpr int GROUPS = kShMergeThreads / (D / 4), REGS = 8;
    __shared__ float wt[kShMergeThreads], red[2][kShMergeThreads / kWave];
    __shared__ f32x4s osum[GROUPS][D / 4];
    const uint32_t qrow = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    if (qrow >= (uint32_t)a.grid.qrows) return;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6, P = a.grid.np + a.grid.nt;
    const int d = 4 * (t % (D / 4)), grp = t / (D / 4);
    const ShParts r = row_parts(a, qrow);
    float M = -INFINITY, L = 0.f;
    f32x4s o = {};
    for (int k0 = 0; k0 < P; k0 += kShMergeThreads) {
        const int np = min(P - k0, kShMergeThreads);
        const float2 e = a.ms[(int64_t)(k0 + min(t, np - 1)) * a.grid.qrows + qrow];
        f32x4s v[REGS];
        const auto sums = [&](int j) {  // of this group's j-th partial
            return *reinterpret_cast<const f32x4s *>(a.acc + ((int64_t)(k0 + min(grp + j * GROUPS, np - 1)) * a.grid.qrows + qrow) * D + d);
        };
#pragma unroll
        for (int j = 0; j < REGS; ++j) v[j] = sums(j);
        const bool mine = t < np && has_part(a, r, k0 + t);
        const float mx = wave_max(mine ? e.x : -INFINITY);
        if (lane == 0) red[0][wv] = mx;
        lds_barrier();
        float nm = M;
#pragma unroll
        for (int w = 0; w < kShMergeThreads / kWave; ++w) nm = fmaxf(nm, red[0][w]);
        const float ref = nm == -INFINITY ? 0.f : nm;
        const float w = mine ? exp2f(e.x - ref) : 0.f;
        wt[t] = mine ? w : -1.f;  // (-1: no partial there)
        const float ws = wave_sum(mine ? e.y * w : 0.f);
        if (lane == 0) red[1][wv] = ws;
        lds_barrier();
        const float sc = exp2f(M - ref);
        L *= sc;
        o *= sc;
#pragma unroll
        for (int w2 = 0; w2 < kShMergeThreads / kWave; ++w2) L += red[1][w2];
        M = nm;
        for (int j0 = 0; grp + j0 * GROUPS < np; j0 += REGS) {
#pragma unroll
            for (int j = 0; j < REGS; ++j) {
                if (j0 > 0) v[j] = sums(j0 + j);
                const int k = grp + (j0 + j) * GROUPS;
                const float w2 = k < np ? wt[k & (kShMergeThreads - 1)] : -1.f;
                if (w2 >= 0.f || w2 != w2) o += v[j] * w2;
            }
        }
        lds_barrier();  // wt and red are free again
    }
    osum[grp][t % (D / 4)] = o;
    __syncthreads();
    if (t < D / 4) {
        for (int g = 1; g < GROUPS; ++g) o += osum[g][t];
        write_out(a, qrow, d, r.bad, M, L, o);
    }
}

template <bool BF, int D>
static void launch_shared(const SharedArgs &a, dim3 grid, hipStream_t st)
{
    if (a.grid.wq == 4) hipLaunchKernelGGL((k_shared<BF, D, 4>), grid, dim3(kShThreads), 0, st, a);
    else if (a.grid.wq == 2) hipLaunchKernelGGL((k_shared<BF, D, 2>), grid, dim3(kShThreads), 0, st, a);
    else hipLaunchKernelGGL((k_shared<BF, D, 1>), grid, dim3(kShThreads), 0, st, a);
}

template <int D>
static void launch_merge(const SharedArgs &a, int few, dim3 grid, hipStream_t st)
{
    const dim3 b(kShMergeThreads);
    if (few == 2) hipLaunchKernelGGL((k_shared_merge_few<D, 2>), grid, b, 0, st, a);
    else if (few == 3) hipLaunchKernelGGL((k_shared_merge_few<D, 3>), grid, b, 0, st, a);
    else if (few == 5) hipLaunchKernelGGL((k_shared_merge_few<D, 5>), grid, b, 0, st, a);
    else if (few == 8) hipLaunchKernelGGL((k_shared_merge_few<D, 8>), grid, b, 0, st, a);
    else if (few == 14) hipLaunchKernelGGL((k_shared_merge_few<D, 14>), grid, b, 0, st, a);
    else if (few == kShFew) hipLaunchKernelGGL((k_shared_merge_few<D, kShFew>), grid, b, 0, st, a);
    else hipLaunchKernelGGL(k_shared_merge<D>, grid, b, 0, st, a);
}

hipError_t shared_launch(SharedArgs a, bool bf16, hipStream_t st)
{
    const auto grid = [](int64_t n) {
        return dim3((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX));
    };
    const int64_t blocks = a.grid.prompt_blocks + (a.grid.tail_waves + kShWaves - 1) / kShWaves;
    if (blocks > 0) {
        const dim3 g = grid(blocks);
        if (bf16 && a.D == 128) ECOKV_TIMED("decode_shared", st, (launch_shared<true, 128>(a, g, st)));
        else if (bf16) ECOKV_TIMED("decode_shared", st, (launch_shared<true, 64>(a, g, st)));
        else if (a.D == 128) ECOKV_TIMED("decode_shared", st, (launch_shared<false, 128>(a, g, st)));
        else ECOKV_TIMED("decode_shared", st, (launch_shared<false, 64>(a, g, st)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int parts = a.grid.np + a.grid.nt;
    const int few = parts <= 2 ? 2 : parts <= 3 ? 3 : parts <= 5 ? 5 : parts <= 8 ? 8 : parts <= 14 ? 14 : parts <= kShFew ? kShFew : 0;
    const int per = few ? kShMergeThreads / (a.D / 4) : 1;
    const dim3 g = grid((a.grid.qrows + per - 1) / per);
    ECOKV_TIMED("shared_merge", st, (a.D == 128 ? launch_merge<128>(a, few, g, st) : launch_merge<64>(a, few, g, st)));
    return hipGetLastError();
}

}  // namespace ecokv
