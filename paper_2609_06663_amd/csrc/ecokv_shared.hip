// ecokv_decode_shared kernels (gfx950): one query of each continuation of a
// batch over its prompt's kept rows and its own paged tail.
//
// For a (layer, KV head) the query rows that read one prompt's rows are its G
// query heads of all the prompt's continuations: M = G n of them, so the rows
// are the operands of matrix products, read once for a tile of query rows
// instead of once for every continuation.  Softmax over both sets of rows: each
// block takes a part of one set for one tile of query rows and leaves (maximum,
// sum, sum of weighted values); k_shared_merge joins a query row's partials by
// their log-sum-exp.
//  * S^T = K Q^T: the rows as A, the query rows as B (v_mfma_f32_16x16x32_bf16,
//    or v_mfma_f32_16x16x4_f32 for fp32 rows).  Lane l holds the logits of rows
//    4 (l / 16) .. +3 of each 16 against query row l % 16.
//  * O^T += V^T P^T: the weights are the B operand in the registers they are
//    computed in: operand element j of lane group g is row 4 g + j of the first
//    16 rows (j < 4) or of the second, and V^T, read transposed from a wave's
//    LDS stage, takes the same order.  Every lane's sums belong to query row
//    l % 16, whose maximum and sum the lane also keeps, so moving the reference
//    costs no exchange.
//  * bf16 rows: a weight enters the product as three bf16 summands (24 bits):
//    rounded to one it would leave 2^-9 of every weight, two leave 2^-17, where
//    the sums beside it are fp32.
#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4s __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8s __attribute__((ext_vector_type(8)));
typedef float f32x4s __attribute__((ext_vector_type(4)));
typedef short s16x4s __attribute__((ext_vector_type(4)));

constexpr int kShThreads = kShWaves * kWave;
constexpr float kShRebase = 8.f;  // log2 headroom of the lazily moved reference

// A block's work: query rows q0 .. q0 + nq - 1 of the nc continuations from c0
// on (row m: head m / nc of the group, continuation c0 + m % nc), rows [row0,
// row0 + rows) of the prompt's unit or of the tail of continuation c0, and the
// part of the workspace that takes the partials.
struct SharedItem {
    int l, h, c0, nc, q0, nq, row0, rows, part;
    int64_t base;  // first row of the prompt's unit
    bool paged;
};

__device__ __forceinline__ bool shared_item(const SharedArgs &a, int64_t b, SharedItem &it)
{
    const SharedGrid &g = a.grid;
    it.paged = b >= g.prompt_blocks;
    int n, parts, lh, part;
    if (!it.paged) {
        const int per = g.tiles * g.np;
        lh = (int)(b / per);
        const int r = (int)(b - (int64_t)lh * per);
        part = r / g.tiles;
        const int tile = r - part * g.tiles;
        int s = 0;
        while (s + 1 < a.B && g.tile0[s + 1] <= tile) ++s;
        it.c0 = a.fan[s];
        it.nc = a.fan[s + 1] - it.c0;
        it.q0 = (tile - g.tile0[s]) * g.qt;
        it.nq = min(g.qt, a.G * it.nc - it.q0);
        const int64_t u = (int64_t)lh * a.B + s;
        n = uniform_i32(a.counts[u]);
        it.base = uniform_i32(a.offsets[u]);
        if (n > a.max_count) n = 0;  // (the merge writes NaN)
        parts = g.np;
        it.part = part;
    } else {
        const int zg = tail_groups(a.G);
        int64_t r = b - g.prompt_blocks;
        if (r >= g.tail_blocks) return false;
        const int64_t per = (int64_t)a.N * zg * g.nt;
        lh = (int)(r / per);
        r -= (int64_t)lh * per;
        const int c = (int)(r / (zg * g.nt)), z = (int)(r - (int64_t)c * (zg * g.nt));
        part = z / zg;
        it.c0 = c;
        it.nc = 1;
        it.q0 = 16 * (z - part * zg);
        it.nq = min(16, a.G - it.q0);
        n = uniform_i32(a.tail_counts[c]);
        if (n > a.max_tail) n = 0;
        it.base = 0;
        parts = g.nt;
        it.part = g.np + part;
    }
    it.l = lh / a.Hkv;
    it.h = lh - it.l * a.Hkv;
    n = max(n, 0);
    const int64_t pr = part_rows(n, parts);
    it.row0 = (int)min(part * pr, (int64_t)n);
    it.rows = (int)min((int64_t)(n - it.row0), pr);
    return it.rows > 0;
}

// Place of 16-byte chunk c of row r of a wave's V stage: the rows' chunks
// permuted so that the transposed reads (bf16: 4 rows of 32 bytes per 16 lanes;
// fp32: 4 rows, 4 apart, of 64 bytes) do not all start at one bank.
template <bool BF, int S>
__device__ __forceinline__ int stage_chunk(int r, int c)
{
    if constexpr (BF) return r * S + (c ^ (r & (S - 1)));
    else return r * S + (c ^ (((r >> 2) & 3) << 2));
}

template <bool BF, int D>
__global__ __launch_bounds__(kShThreads) void k_shared(SharedArgs a)
{
    constexpr int RB = D * (BF ? 2 : 4);   // row bytes
    constexpr int S = RB / 16;             // 16-byte chunks per row
    constexpr int SUB = BF ? 2 : 1;        // 16-row groups per tile
    constexpr int TR = 16 * SUB;           // rows per tile
    constexpr int KS = RB / 64;            // K operand loads per 16 rows
    constexpr int RPI = kWave / S;         // V rows per load instruction
    constexpr int NV = TR / RPI;
    constexpr int DT = D / 16;             // 16-dimension tiles of the output
    constexpr int STAGE = TR * S;          // chunks of a wave's stage
    constexpr int OUTF = 16 * D;           // floats of a wave's sums
    static_assert(STAGE * 16 <= OUTF * 4, "the stages and the waves' sums share LDS");
    __shared__ __attribute__((aligned(16))) float lds[kShWaves][OUTF];
    __shared__ float wm[kShWaves][16], wl[kShWaves][16];

    SharedItem it;
    if (!shared_item(a, (int64_t)blockIdx.z * kGridX + blockIdx.x, it)) return;
    const int lane = threadIdx.x & 63, wv = uniform_i32(threadIdx.x >> 6);
    const int r16 = lane & 15, kg = lane >> 4, seg = lane % S, rg = lane / S;

    // this wave's rows of the block's part
    const int quarter = ((it.rows + kShWaves - 1) / kShWaves + kShTile - 1) / kShTile * kShTile;
    const int w0 = it.row0 + wv * quarter;
    const int nrows = max(0, min(it.row0 + it.rows - w0, quarter));

    // address of row r of this wave's (clamped into its rows), and whether its page is one
    const auto row_at = [&](const char *prompt, const char *tail, int r, bool &bad) -> const char * {
        const int row = w0 + min(r, nrows - 1);
        if (!it.paged) return prompt + (it.base + row) * RB;
        const int page = tail_page(a.map, it.c0, row);
        bad = page < 0;
        return tail + tail_row(a.map, a.Hkv, it.l, it.h, max(page, 0), row) * RB;
    };

    // the query rows as operand B (rows past nq repeat the last)
    u32x4s qb[KS];
    {
        const int m = it.q0 + min(r16, it.nq - 1), g = m / it.nc, c = it.c0 + m % it.nc;
        const char *q = a.Q + (((int64_t)it.l * a.Hq + it.h * a.G + g) * a.N + c) * RB + 16 * kg;
#pragma unroll
        for (int st = 0; st < KS; ++st) qb[st] = *reinterpret_cast<const u32x4s *>(q + 64 * st);
    }
    float m = -INFINITY, ls = 0.f;
    f32x4s acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = (f32x4s){0.f, 0.f, 0.f, 0.f};
    u32x4s *const stage = reinterpret_cast<u32x4s *>(&lds[wv][0]);

    for (int b0 = 0; b0 < nrows; b0 += TR) {
        u32x4s kx[SUB][KS], vx[NV];
        bool bad[SUB], unused = false;
#pragma unroll
        for (int t = 0; t < SUB; ++t) {
            bad[t] = false;
            const char *p = row_at(a.Kc, a.Kt, b0 + 16 * t + r16, bad[t]) + 16 * kg;
#pragma unroll
            for (int st = 0; st < KS; ++st) kx[t][st] = *reinterpret_cast<const u32x4s *>(p + 64 * st);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int r = b0 + RPI * i + rg;
            vx[i] = *reinterpret_cast<const u32x4s *>(row_at(a.Vc, a.Vt, r, unused) + 16 * seg);
            if (r >= nrows) vx[i] = (u32x4s){0u, 0u, 0u, 0u};  // (a row that is not there may hold no infinity)
        }
        f32x4s x[SUB];
#pragma unroll
        for (int t = 0; t < SUB; ++t) {
            x[t] = (f32x4s){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                if constexpr (BF) {
                    x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8s, kx[t][st]),
                                                                   __builtin_bit_cast(bf16x8s, qb[st]), x[t], 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kx[t][st][e]),
                                                                    __uint_as_float(qb[st][e]), x[t], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) stage[stage_chunk<BF, S>(RPI * i + rg, seg)] = vx[i];
        float mb = -INFINITY;
#pragma unroll
        for (int t = 0; t < SUB; ++t) {
            // rows of bad pages, as lane r16 of each lane group found them
            const unsigned badm = it.paged ? (unsigned)(__builtin_amdgcn_ballot_w64(bad[t]) & 0xffffu) : 0u;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int k = 4 * kg + r;
                x[t][r] = b0 + 16 * t + k < nrows ? ((badm >> k) & 1u ? NAN : x[t][r] * a.qscale) : -INFINITY;
                mb = fmaxf(mb, x[t][r]);
            }
        }
        mb = across32(across16(mb, OpMax{}), OpMax{});
        const bool move = mb > m + kShRebase;  // (from m = -inf: with the first finite logit)
        if (__builtin_amdgcn_ballot_w64(move)) {
            const float nm = move ? mb : m;
            const float sc = __builtin_amdgcn_exp2f(m - nm);  // 0 while m = -inf
            const float s1 = move ? sc : 1.f;
            ls *= s1;
            m = nm;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[d][r] *= s1;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int t = 0; t < SUB; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[t][r] = __builtin_amdgcn_exp2f(x[t][r] - ref);
                ls += x[t][r];
            }
        // (a wave's own LDS accesses are ordered)
        if constexpr (BF) {
            bf16x8s p[3];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y = x[j >> 2][j & 3];
#pragma unroll
                for (int s = 0; s < 3; ++s) {
                    p[s][j] = (__bf16)y;
                    y -= (float)p[s][j];
                }
            }
            const uint16_t *st16 = reinterpret_cast<const uint16_t *>(stage);
            const int tr = 4 * kg + (r16 >> 2), tb = r16 & 3;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int c = 2 * d + (tb >> 1), off = (tb & 1) * 4;
                s16x4s v[2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4s *)(
                        const_cast<uint16_t *>(st16 + 8 * stage_chunk<BF, S>(16 * t + tr, c) + off)));
                const short __attribute__((ext_vector_type(8))) v8 = {v[0][0], v[0][1], v[0][2], v[0][3],
                                                                      v[1][0], v[1][1], v[1][2], v[1][3]};
#pragma unroll
                for (int s = 2; s >= 0; --s)
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8s, v8), p[s], acc[d], 0, 0, 0);
            }
        } else {
            const float *st32 = reinterpret_cast<const float *>(stage);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = st32[4 * stage_chunk<BF, S>(4 * kg + r, 4 * d + (r16 >> 2)) + (r16 & 3)];
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[0][r], acc[d], 0, 0, 0);
                }
        }
    }

    ls = across32(across16(ls, OpAdd{}), OpAdd{});
    if (lane < 16) {
        wm[wv][lane] = m;
        wl[wv][lane] = ls;
    }
    // (the wave's stage has been read: its sums take its place)
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4s *>(&lds[wv][r16 * D + 16 * d + 4 * kg]) = acc[d];
    __syncthreads();
    for (int e = threadIdx.x; e < it.nq * D; e += kShThreads) {
        const int q = e / D, d = e - q * D;
        float M = wm[0][q];
        for (int w = 1; w < kShWaves; ++w) M = fmaxf(M, wm[w][q]);
        const float ref = M == -INFINITY ? 0.f : M;
        float L = 0.f, A = 0.f;
        for (int w = 0; w < kShWaves; ++w) {
            const float wt = exp2f(wm[w][q] - ref);
            L += wl[w][q] * wt;
            A += lds[w][q * D + d] * wt;
        }
        const int mq = it.q0 + q;
        const int64_t row = (int64_t)it.part * a.grid.qrows +
                            ((int64_t)it.l * a.Hq + it.h * a.G + mq / it.nc) * a.N + it.c0 + mq % it.nc;
        a.acc[row * D + d] = A;
        if (d == 0) a.ms[row] = make_float2(M, L);
    }
}

// One block per query row: its prompt parts and tail parts joined.
template <int D>
__global__ __launch_bounds__(D) void k_shared_merge(SharedArgs a)
{
    const int64_t qrow = (int64_t)blockIdx.z * kGridX + blockIdx.x;
    if (qrow >= a.grid.qrows) return;
    const int c = (int)(qrow % a.N), q = (int)((qrow / a.N) % a.Hq), l = (int)(qrow / ((int64_t)a.N * a.Hq));
    int s = 0;
    while (s + 1 < a.B && a.fan[s + 1] <= c) ++s;
    int np = 0, nt = 0;
    bool bad = false;
    if (a.max_count > 0) {
        const int n = uniform_i32(a.counts[((int64_t)l * a.Hkv + q / a.G) * a.B + s]);
        bad = n < 0 || n > a.max_count;
        np = bad ? 0 : parts_used(n, a.grid.np);
    }
    if (a.max_tail > 0) {
        const int n = uniform_i32(a.tail_counts[c]);
        const bool b2 = n < 0 || n > a.max_tail;
        nt = b2 ? 0 : parts_used(n, a.grid.nt);
        bad = bad || b2;
    }
    const int d = threadIdx.x;
    float M = -INFINITY, L = 0.f, o = 0.f;
    for (int k = 0; k < np + nt; ++k) {
        const int64_t row = (int64_t)(k < np ? k : a.grid.np + k - np) * a.grid.qrows + qrow;
        const float2 e = a.ms[row];
        const float v = a.acc[row * D + d];
        const float nm = fmaxf(M, e.x), ref = nm == -INFINITY ? 0.f : nm;
        const float f = exp2f(M - ref), w = exp2f(e.x - ref);  // 0 from -inf
        L = L * f + e.y * w;
        o = o * f + v * w;
        M = nm;
    }
    a.O[qrow * D + d] = bad ? NAN : (L == 0.f ? 0.f : o / L);
    if (d == 0 && a.lse) a.lse[qrow] = bad ? NAN : (L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f);
}

hipError_t shared_launch(SharedArgs a, bool bf16, hipStream_t st)
{
    const auto grid = [](int64_t n) {
        return dim3((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX));
    };
    const int64_t blocks = a.grid.prompt_blocks + a.grid.tail_blocks;
    if (blocks > 0) {
        const dim3 g = grid(blocks), b(kShThreads);
        if (bf16 && a.D == 128) ECOKV_TIMED("decode_shared", st, hipLaunchKernelGGL((k_shared<true, 128>), g, b, 0, st, a));
        else if (bf16) ECOKV_TIMED("decode_shared", st, hipLaunchKernelGGL((k_shared<true, 64>), g, b, 0, st, a));
        else if (a.D == 128) ECOKV_TIMED("decode_shared", st, hipLaunchKernelGGL((k_shared<false, 128>), g, b, 0, st, a));
        else ECOKV_TIMED("decode_shared", st, hipLaunchKernelGGL((k_shared<false, 64>), g, b, 0, st, a));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 g = grid(a.grid.qrows);
    if (a.D == 128) ECOKV_TIMED("shared_merge", st, hipLaunchKernelGGL(k_shared_merge<128>, g, dim3(128), 0, st, a));
    else ECOKV_TIMED("shared_merge", st, hipLaunchKernelGGL(k_shared_merge<64>, g, dim3(64), 0, st, a));
    return hipGetLastError();
}

}  // namespace ecokv
