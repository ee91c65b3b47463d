// ecokv_accumulate kernel (gfx950): every cache row's attention weight, summed over
// the query rows that see it and added to what the row had before.
//
//   out[j] = decay in[j] + sum over heads g of the group and queries i of
//            exp(q_i . k_j / sqrt(D) - lse_i)
//
// The log-sum-exp is the one that the attention left, so one pass over K is
// enough, and a row's sum needs no other row: a wave keeps its rows in registers
// (as the B operand of v_mfma_f32_16x16x32_bf16 or v_mfma_f32_16x16x4_f32) and
// takes the query rows 16 at a time (A), which come from L2.  A lane then holds the
// logits of four query rows against one cache row, adds up their weights, and the
// four lanes of a row join their sums at the end.  No atomics: a call gives the same
// bits again.
#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4m __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8m __attribute__((ext_vector_type(8)));
typedef float f32x4m __attribute__((ext_vector_type(4)));

constexpr int kMassThreads = kMassWaves * kWave;
constexpr int kMassList = 64 * 64;  // queries that a block lists at a time: 64 continuations of 64 nodes

template <bool BF, int D>
struct MassGeo {
    static constexpr int RB = D * (BF ? 2 : 4);  // row bytes
    static constexpr int ST = RB / 64;           // 16-byte operands of a row per lane
};

// Logits (unscaled) of 16 query rows against 16 cache rows: query row 4 (lane / 16) + r
// of cache row lane % 16.
template <bool BF, int D>
__device__ __forceinline__ f32x4m mass_logits(const u32x4m (&q)[MassGeo<BF, D>::ST], const u32x4m (&k)[MassGeo<BF, D>::ST])
{
    if constexpr (BF) {
        f32x4m x = {};
#pragma unroll
        for (int s = 0; s < MassGeo<BF, D>::ST; ++s)
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8m, q[s]), __builtin_bit_cast(bf16x8m, k[s]), x, 0, 0, 0);
        return x;
    } else {
        f32x4m y[4] = {};
#pragma unroll
        for (int s = 0; s < MassGeo<BF, D>::ST; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[s][e]), __uint_as_float(k[s][e]), y[e], 0, 0, 0);
        return (y[0] + y[1]) + (y[2] + y[3]);
    }
}

template <bool BF, int D, int RT>
__global__ __launch_bounds__(kMassThreads) void k_mass(MassArgs a)
{
    typedef MassGeo<BF, D> Ge;
    constexpr int ROWS = 16 * RT;  // of a wave
    __shared__ int list[kMassList];
    __shared__ int listed;
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
    const int first_row = (int)(part * (uint32_t)(ROWS * kMassWaves));
    if (first_row >= n) return;
    const int l = (int)((uint32_t)lh / (uint32_t)a.Hkv), h = lh - l * a.Hkv;
    const int row0 = first_row + wv * ROWS;

    // this lane's rows (row16 of every tile; past the end: the last) and where they are
    u32x4m k[RT][Ge::ST];
    int64_t place = -1;  // of the mass of row grp of the tiles, -1 for none
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = row0 + 16 * t + row16, in = min(r, n - 1);
        int64_t at = base + in;
        bool there = r < n;
        if (tail) {
            const int page = tail_page(a.map, c0, in);
            there = there && page >= 0;
            at = tail_row(a.map, a.Hkv, l, h, max(page, 0), in);
        }
        const char *p = (tail ? a.Kt : a.Kc) + at * Ge::RB + 16 * grp;
#pragma unroll
        for (int s = 0; s < Ge::ST; ++s) k[t][s] = *reinterpret_cast<const u32x4m *>(p + 64 * s);
        if (t == grp && there) place = at;
    }

    float sum[RT] = {};
    // the accepted ones of a path: the k-th sees the tail's rows up to its own
    const auto accepted = [&](int c) {
        if (!a.path) return 1;
        const int x = a.accepted[c];
        return x < 0 || x > a.nodes ? 0 : x;
    };
    const int fresh = tail ? accepted(c0) : 0;  // rows at the end that are new
    for (int cc = c0; cc < c1; cc += 64) {
        const int nc = min(c1 - cc, 64);
        int pairs = nc;  // (continuation, place in its path)
        if (a.path) {
            __syncthreads();
            if (wv == 0) {
                const int x = lane < nc ? accepted(cc + lane) : 0;
                const int end = (int)wave_incl_scan((uint32_t)x);
                for (int j = 0; j < x; ++j) {
                    const int node = a.path[(int64_t)(cc + lane) * a.nodes + j];
                    list[end - x + j] = node < 0 || node >= a.nodes ? -1 : (cc + lane) * a.nodes + node;
                }
                if (lane == 63) listed = end;
            }
            __syncthreads();
            pairs = uniform_i32(listed);
        }
        const int queries = pairs * a.G;
        for (int q0 = 0; q0 < queries; q0 += 16) {
            const int i = min(q0 + row16, queries - 1);
            const int p = (int)((uint32_t)i / (uint32_t)a.G), g = i - p * a.G;
            const int node = a.path ? list[p] : cc + p;
            const int64_t qrow = ((int64_t)l * a.Hq + h * a.G + g) * ((int64_t)a.N * a.nodes) + max(node, 0);
            u32x4m q[Ge::ST];
            const char *qp = a.Q + qrow * Ge::RB + 16 * grp;
#pragma unroll
            for (int s = 0; s < Ge::ST; ++s) q[s] = *reinterpret_cast<const u32x4m *>(qp + 64 * s);
            // a query that is not there, or that saw no row, weighs nothing
            float lse = a.lse[qrow];
            if (node < 0 || q0 + row16 >= queries || lse == -INFINITY) lse = INFINITY;
            const int last = tail ? n - fresh + p : 0;  // the last row that it sees
            float z[4], dz[4];
            int see[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                z[r] = __shfl(lse, 4 * grp + r, kWave);
                see[r] = __shfl(last, 4 * grp + r, kWave);
                dz[r] = fabsf(z[r]) < INFINITY ? z[r] * a.scale_rest : 0.f;
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const f32x4m x = mass_logits<BF, D>(q, k[t]);
                const int row = row0 + 16 * t + row16;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // x / sqrt(D) - lse: the scale's rounding, times x, is that times lse where the weight counts
                    const float e = fmaf(x[r], a.scale, -z[r]) + dz[r];
                    const float w = __builtin_amdgcn_exp2f(e * 1.4426950408889634f);
                    sum[t] += !tail || row <= see[r] ? w : 0.f;
                }
            }
        }
    }
    float mine = 0.f;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const float s = across32(across16(sum[t], OpAdd{}), OpAdd{});
        if (t == grp) mine = s;
    }
    if (place >= 0) {
        const float *in = tail ? a.tail_mass : a.mass;
        float *out = tail ? a.tail_mass_out : a.mass_out;
        const int row = row0 + 16 * grp + row16;
        out[place] = tail && row >= n - fresh ? mine : fmaf(a.decay, in[place], mine);
    }
}

template <bool BF, int D>
static void launch_mass(const MassArgs &a, dim3 grid, hipStream_t st)
{
    if (a.rt == 4) hipLaunchKernelGGL((k_mass<BF, D, 4>), grid, dim3(kMassThreads), 0, st, a);
    else hipLaunchKernelGGL((k_mass<BF, D, 2>), grid, dim3(kMassThreads), 0, st, a);
}

hipError_t mass_launch(const MassArgs &a, bool bf16, hipStream_t st)
{
    const int64_t n = a.kept_blocks + a.tail_blocks;
    if (n == 0) return hipSuccess;
    const dim3 g((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX));
    if (bf16 && a.D == 128) ECOKV_TIMED("accumulate", st, (launch_mass<true, 128>(a, g, st)));
    else if (bf16) ECOKV_TIMED("accumulate", st, (launch_mass<true, 64>(a, g, st)));
    else if (a.D == 128) ECOKV_TIMED("accumulate", st, (launch_mass<false, 128>(a, g, st)));
    else ECOKV_TIMED("accumulate", st, (launch_mass<false, 64>(a, g, st)));
    return hipGetLastError();
}

}  // namespace ecokv
