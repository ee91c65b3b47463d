// ecokv_accumulate kernel (gfx950): every cache row's attention weight, summed over
// the query rows that see it and added to what the row had before.
//
//   out[j] = decay in[j] + sum over heads g of the group and queries i of
//            exp(q_i . k_j / sqrt(D) - lse_i)
//
// The log-sum-exp is the one that the attention left, so one pass over K is
// enough, and a row's sum needs no other row: a wave keeps its rows in registers
// (as the A operand of v_mfma_f32_16x16x32_bf16 or v_mfma_f32_16x16x4_f32) and
// takes the query rows 16 at a time (B), which the block stages in LDS.  A lane then holds the
// logits of one query row against four cache rows of every tile and adds up their
// weights; the 16 lanes of a row join their sums at the end.  (The other way round
// every query tile had to hand its log-sum-exps to the lanes.)  No atomics: a call
// gives the same bits again.
//
// A weight is exp2(x c - z), c = log2 e / sqrt(D) and z = lse log2 e: both are rounded,
// and z is the larger of the two by far, so what the roundings leave out (of c, times
// z where the weight counts) is added to the difference: four instructions a weight.
#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4m __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8m __attribute__((ext_vector_type(8)));
typedef float f32x4m __attribute__((ext_vector_type(4)));

constexpr int kMassThreads = kMassWaves * kWave;
constexpr int kMassList = 64 * 64;  // nodes that a block lists at a time: 64 continuations of 64
// Tiles of 16 query rows staged at a time: with rows of up to 256 bytes six leave room for
// four blocks on a compute unit (34 KB of LDS each; with 512, fp32 of 128, 58 KB and two)
// and take 96 rows for all of a block's pieces at once (us, accepted paths of four
// continuations, 28 layers, bf16 of 128: four tiles 74.6, six 56.4, eight 62.8).
constexpr int kMassTiles = 6;

template <bool BF, int D>
struct MassGeo {
    static constexpr int RB = D * (BF ? 2 : 4);  // row bytes
    static constexpr int ST = RB / 64;           // 16-byte operands of a row per lane
};

// Logits (unscaled) of 16 cache rows against 16 query rows: cache row 4 (lane / 16) + r,
// query row lane % 16.
template <bool BF, int D>
__device__ __forceinline__ f32x4m mass_logits(const u32x4m (&k)[MassGeo<BF, D>::ST], const u32x4m (&q)[MassGeo<BF, D>::ST])
{
    if constexpr (BF) {
        f32x4m x = {};
#pragma unroll
        for (int s = 0; s < MassGeo<BF, D>::ST; ++s)
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8m, k[s]), __builtin_bit_cast(bf16x8m, q[s]), x, 0, 0, 0);
        return x;
    } else {
        f32x4m y[4] = {};
#pragma unroll
        for (int s = 0; s < MassGeo<BF, D>::ST; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[s][e]), __uint_as_float(q[s][e]), y[e], 0, 0, 0);
        return (y[0] + y[1]) + (y[2] + y[3]);
    }
}

template <bool BF, int D>
__global__ __launch_bounds__(kMassThreads, BF ? 4 : 3) void k_mass(MassArgs a)
{
    typedef MassGeo<BF, D> Ge;
    constexpr int RT = kMassRows / 16, ROWS = kMassRows;  // of a wave
    __shared__ uint16_t list[kMassList];              // nodes, counted from the first listed continuation's; 65535: none
    __shared__ u32x4m qs[kMassTiles][Ge::ST][kWave];  // 16 query rows each, in the order of the operands
    __shared__ float zs[2][16 * kMassTiles];          // z, and what its roundings leave out
    __shared__ int lasts[16 * kMassTiles];            // the last row of the tail that a query sees; INT32_MIN: it weighs nothing
    __shared__ int voids[kMassTiles];                 // whether a tile has such queries
    const uint32_t b = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    const int lane = threadIdx.x & 63, wv = uniform_i32(threadIdx.x >> 6), grp = lane >> 4, row16 = lane & 15;
    const bool tail = b >= (uint32_t)a.kept_blocks;
    // the unit, its rows, its continuations
    int lh, n, c0, c1;
    uint32_t part;
    int64_t base = 0;
    if (!tail) {
        if (a.kept_parts == 0) return;
        const uint32_t u = b / (uint32_t)a.kept_parts;
        part = b - u * (uint32_t)a.kept_parts;
        lh = (int)(u / (uint32_t)a.B);
        const int s = (int)(u - (uint32_t)lh * (uint32_t)a.B);
        n = uniform_i32(a.counts[u]);
        if (n > a.max_count) n = 0;  // (counts out of their bounds: left alone)
        base = uniform_i32(a.offsets[u]);
        c0 = a.fan[s], c1 = a.fan[s + 1];
    } else {
        const uint32_t t = b - (uint32_t)a.kept_blocks;
        if (t >= (uint32_t)a.tail_blocks) return;
        const uint32_t f = t / (uint32_t)a.tail_parts;
        part = t - f * (uint32_t)a.tail_parts;
        lh = (int)(f / (uint32_t)a.N);
        c0 = (int)(f - (uint32_t)lh * (uint32_t)a.N), c1 = c0 + 1;
        n = uniform_i32(a.tail_counts[c0]);
        if (n > a.max_tail) n = 0;
    }
    constexpr int BLOCK = ROWS * kMassWaves;
    const int64_t stride = (int64_t)(tail ? a.tail_parts : a.kept_parts) * BLOCK;
    if ((int64_t)part * BLOCK >= n) return;
    const int l = (int)((uint32_t)lh / (uint32_t)a.Hkv), h = lh - l * a.Hkv;
    const float *const in = tail ? a.tail_mass : a.mass;
    float *const out = tail ? a.tail_mass_out : a.mass_out;
    // the accepted ones of a path: the k-th sees the tail's rows up to its own
    const auto accepted = [&](int c) {
        if (!a.path) return 1;
        const int x = a.accepted[c];
        return x < 0 || x > a.nodes ? 0 : x;
    };
    const int fresh = tail ? accepted(c0) : 0;  // rows at the end that are new
    // The accepted nodes of up to 64 continuations from cc on, one after the other, into
    // the list: a thread for each place of a path (a loop over a path's places waited for
    // each of them).  Returns their number.
    const auto enlist = [&](int cc, int nc) {
        const int x = lane < nc ? accepted(cc + lane) : 0;
        const int end = (int)wave_incl_scan((uint32_t)x);
        __syncthreads();  // (the list is free)
        for (int e = 0; e < nc * a.nodes; e += kMassThreads) {
            const int i = min(e + (int)threadIdx.x, nc * a.nodes - 1);
            const int c = (int)((uint32_t)i / (uint32_t)a.nodes), k = i - c * a.nodes;
            const int xc = __shfl(x, c, kWave), ec = __shfl(end, c, kWave);
            if (k < xc) {
                const int node = a.path[(int64_t)(cc + c) * a.nodes + k];
                list[ec - xc + k] = (uint16_t)(node < 0 || node >= a.nodes ? 65535 : c * a.nodes + node);
            }
        }
        __syncthreads();
        return (int)__builtin_amdgcn_readlane(end, 63);
    };
    // Query rows qb .. of the listed pairs (continuation, node), a wave 16 of them at a time.
    const auto stage = [&](int cc, int queries, int qb) {
        __syncthreads();  // (nobody reads what was staged before)
        for (int qt = wv; qt < kMassTiles && qb + 16 * qt < queries; qt += kMassWaves) {
            const int q0 = qb + 16 * qt, i = min(q0 + row16, queries - 1);
            const int p = (int)((uint32_t)i / (uint32_t)a.G), g = i - p * a.G;
            const int entry = a.path ? list[p] : p;
            const bool none = entry == 65535 && a.path;
            const int64_t qrow = ((int64_t)l * a.Hq + h * a.G + g) * ((int64_t)a.N * a.nodes) + (int64_t)cc * a.nodes + (none ? 0 : entry);
            const char *qp = a.Q + qrow * Ge::RB + 16 * grp;
            u32x4m q[Ge::ST];
#pragma unroll
            for (int s = 0; s < Ge::ST; ++s) q[s] = *reinterpret_cast<const u32x4m *>(qp + 64 * s);
            float lse = a.lse[qrow];
#pragma unroll
            for (int s = 0; s < Ge::ST; ++s) qs[qt][s][lane] = q[s];
            // a query that is not there, or that saw no row, weighs nothing, whatever it holds
            const bool nothing = none || q0 + row16 >= queries || lse == -INFINITY;
            const bool odd = __builtin_amdgcn_ballot_w64(nothing) != 0;
            if (lane == 0) voids[qt] = odd;
            constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f;
            const float z = lse * kLog2e;
            if (grp == 0) {
                zs[0][16 * qt + row16] = z;
                zs[1][16 * qt + row16] = fabsf(z) < INFINITY ? z * a.scale_rest - fmaf(lse, kLog2eRest, fmaf(lse, kLog2e, -z)) : 0.f;
                lasts[16 * qt + row16] = nothing ? INT32_MIN : tail ? n - fresh + p : 0;
            }
        }
        __syncthreads();
    };
    // where they fit, one list and one stage serve all of the block's rows
    const int all = c1 - c0 > 64 ? INT32_MAX : (a.path ? enlist(c0, c1 - c0) : c1 - c0) * a.G;
    const bool once = all <= 16 * kMassTiles;
    if (once && all > 0) stage(c0, all, 0);

    for (int64_t first = (int64_t)part * BLOCK; first < n; first += stride) {
        const int row0 = (int)first + wv * ROWS;
        // this lane's rows (row16 of every tile; past the end: the last)
        u32x4m k[RT][Ge::ST];
        const auto where = [&](int64_t r, bool &there) {
            const int row = (int)min(r, (int64_t)n - 1);
            there = r < n;
            if (!tail) return base + row;
            const int page = tail_page(a.map, c0, row);
            there = there && page >= 0;
            return tail_row(a.map, a.Hkv, l, h, max(page, 0), row);
        };
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            bool there;
            const char *p = (tail ? a.Kt : a.Kc) + where((int64_t)row0 + 16 * t + row16, there) * Ge::RB + 16 * grp;
#pragma unroll
            for (int s = 0; s < Ge::ST; ++s) k[t][s] = *reinterpret_cast<const u32x4m *>(p + 64 * s);
        }
        // the row whose sum it writes: row16 % 4 of its four rows of tile row16 / 4
        const int64_t mine_row = (int64_t)row0 + 16 * (row16 >> 2) + 4 * grp + (row16 & 3);
        bool writes;
        const int64_t place = where(mine_row, writes);
        writes = writes && row16 < 4 * RT;
        const float had = in[place];  // (read ahead)
        // a tile with rows that not every query sees
        const bool cut = tail && fresh > 1 && (int64_t)row0 + ROWS > n - fresh + 1;
        float sum[RT][4] = {};
        for (int cc = c0; cc < c1; cc += 64) {
            const int nc = min(c1 - cc, 64);
            const int queries = once || all != INT32_MAX ? all : (a.path ? enlist(cc, nc) : nc) * a.G;
            for (int qb = 0; qb < queries; qb += 16 * kMassTiles) {
                if (!once) stage(cc, queries, qb);
                for (int qt = 0; qt < kMassTiles && qb + 16 * qt < queries; ++qt) {
                    u32x4m q[Ge::ST];
#pragma unroll
                    for (int s = 0; s < Ge::ST; ++s) q[s] = qs[qt][s][lane];
                    const float z = zs[0][16 * qt + row16], dz = zs[1][16 * qt + row16];
                    const int last = lasts[16 * qt + row16];
                    const bool odd = uniform_i32(voids[qt]) != 0;
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const f32x4m x = mass_logits<BF, D>(k[t], q);
                        float w[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale, -z) + dz);
                        if (odd) {  // (a branch: few tiles have such)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (last == INT32_MIN) w[r] = 0.f;
                        }
                        if (cut) {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (row0 + 16 * t + 4 * grp + r > last) w[r] = 0.f;
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[t][r] += w[r];
                    }
                }
            }
        }
        float mine = 0.f;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float s = seg16_sum(sum[t][r]);
                if (row16 == 4 * t + r) mine = s;
            }
        if (writes) out[place] = tail && mine_row >= n - fresh ? mine : fmaf(a.decay, had, mine);
    }
}

hipError_t mass_launch(const MassArgs &a, bool bf16, hipStream_t st)
{
    const int64_t n = a.kept_blocks + a.tail_blocks;
    if (n == 0) return hipSuccess;
    const dim3 g((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX));
    if (bf16 && a.D == 128) ECOKV_TIMED("accumulate", st, hipLaunchKernelGGL((k_mass<true, 128>), g, dim3(kMassThreads), 0, st, a));
    else if (bf16) ECOKV_TIMED("accumulate", st, hipLaunchKernelGGL((k_mass<true, 64>), g, dim3(kMassThreads), 0, st, a));
    else if (a.D == 128) ECOKV_TIMED("accumulate", st, hipLaunchKernelGGL((k_mass<false, 128>), g, dim3(kMassThreads), 0, st, a));
    else ECOKV_TIMED("accumulate", st, hipLaunchKernelGGL((k_mass<false, 64>), g, dim3(kMassThreads), 0, st, a));
    return hipGetLastError();
}

}  // namespace ecokv
