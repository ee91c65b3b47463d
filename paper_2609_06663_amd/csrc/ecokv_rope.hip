// Norms and rotary positions (gfx950): ecokv_prefill_rope for a prompt's
// queries and keys, ecokv_append for the tokens that continue it.
//
// A row x [D] of a token at position p: x <- x / sqrt(mean x^2 + eps) w, then
// each pair (a, b) of rotated dimensions turns by p freq[i].  Every row is read
// and written once, so the calls are bound by HBM for prompts and by the
// latency of one launch for single tokens.
//
// A block takes a few tokens with all their heads: the cosines and sines of a
// token (rot_dim / 2 of each) are computed once, into LDS, and serve its
// H_q + H_kv rows.  A row lies in S = row bytes / 16 lanes, 16 bytes each; the
// half-split layout's other dimension of a pair comes from the lane half a
// rotation away, the interleaved one's from the same lane.
#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4r __attribute__((ext_vector_type(4)));

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;  // tokens per block at most
constexpr int kRopeRows = 4;    // rows a thread has in flight

template <bool BF>
__device__ __forceinline__ void unpack_row(const u32x4r &x, float (&f)[BF ? 8 : 4])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if constexpr (BF) {
            f[2 * c] = __uint_as_float(x[c] << 16);
            f[2 * c + 1] = __uint_as_float(x[c] & 0xffff0000u);
        } else {
            f[c] = __uint_as_float(x[c]);
        }
    }
}
template <bool BF>
__device__ __forceinline__ u32x4r pack_row(const float (&f)[BF ? 8 : 4])
{
    u32x4r x;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if constexpr (BF) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            x[c] = __builtin_bit_cast(unsigned, (bf16x2){(__bf16)f[2 * c], (__bf16)f[2 * c + 1]});
        } else {
            x[c] = __float_as_uint(f[c]);
        }
    }
    return x;
}

// cos and sin of p w.  The angle is p w in turns, reduced to [-1/2, 1/2] in 64
// bits (the product of a 31-bit position and a 24-bit frequency needs more than
// 32 bits to keep its fraction), the rest in 32.
__device__ __forceinline__ float2 turn(int p, float w, float factor)
{
    const double t = (double)p * (double)w * 0.15915494309189533577;
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    return make_float2(factor * c, factor * s);
}

// What a block knows of each of its tokens.
struct TokenPlace {
    int64_t win;  // prefill: row of Q_win of head 0 (a head is B w rows on), or -1
    int64_t tail; // append: row of the tails of head 0 (a head is page_size rows on), or -1
    int l, t;     // layer and token
};

template <bool BF, int D, bool APPEND>
__global__ __launch_bounds__(kRopeThreads) void k_rope(RopeArgs a)
{
    constexpr int EL = BF ? 8 : 4;        // elements per lane
    constexpr int RB = D * (BF ? 2 : 4);  // row bytes
    constexpr int S = RB / 16;            // lanes per row
    constexpr int RPI = kRopeThreads / S; // rows per block and instruction
    __shared__ float2 cs[kRopeTokens][D / 2];
    __shared__ float wt[2][D];
    __shared__ TokenPlace place[kRopeTokens];
    const int64_t first = ((int64_t)blockIdx.z * kGridX + blockIdx.x) * a.per_block;
    const int64_t all = (int64_t)a.L * a.n;
    const int tokens = (int)max((int64_t)0, min((int64_t)a.per_block, all - first));
    if (tokens == 0) return;
    const int tid = threadIdx.x, half = a.rot >> 1;
    const auto position = [&](int64_t ft) {
        const int t = (int)(ft % a.n);
        if (APPEND || a.positions) return a.positions[t];
        int s = 0;
        while (s + 1 < a.B && a.seq.cu[s + 1] <= t) ++s;
        return t - a.seq.cu[s];
    };
    for (int e = tid; e < tokens * half; e += kRopeThreads) {
        const int k = e / half, i = e - k * half;
        cs[k][i] = turn(position(first + k), a.freq[i], a.factor);
    }
    for (int e = tid; e < 2 * D; e += kRopeThreads) {
        const void *w = e < D ? a.qw : a.kw;
        const int d = e < D ? e : e - D;
        if (w) wt[e >= D][d] = BF ? __uint_as_float((unsigned)static_cast<const uint16_t *>(w)[d] << 16) : static_cast<const float *>(w)[d];
    }
    if (tid < tokens) {
        TokenPlace p;
        const int64_t ft = first + tid;
        p.l = (int)(ft / a.n);
        p.t = (int)(ft - (int64_t)p.l * a.n);
        p.win = p.tail = -1;
        if constexpr (APPEND) {
            const int row = a.rows[p.t], page = tail_page(a.map, a.conts ? a.conts[p.t] : p.t, row);
            if (page >= 0) p.tail = tail_row(a.map, a.Hkv, p.l, 0, page, row);
        } else if (a.win) {
            int s = 0;
            while (s + 1 < a.B && a.seq.cu[s + 1] <= p.t) ++s;
            const int j = p.t - (a.seq.cu[s + 1] - a.w);
            if (j >= 0) p.win = ((int64_t)p.l * a.Hq * a.B + s) * a.w + j;
        }
        place[tid] = p;
    }
    __syncthreads();

    const int H = a.hq + a.hk + (APPEND ? a.hk : 0), rows = tokens * H;
    const int seg = tid % S, e0 = seg * EL;
    for (int r0 = tid / S; r0 < (rows + RPI - 1) / RPI * RPI; r0 += RPI * kRopeRows) {
        u32x4r x[kRopeRows];
        int tok[kRopeRows], head[kRopeRows];
#pragma unroll
        for (int j = 0; j < kRopeRows; ++j) {
            const int r = min(r0 + j * RPI, rows - 1);  // (lanes of rows past the last load it again)
            tok[j] = r / H;
            head[j] = r - tok[j] * H;
            const int64_t ft = first + tok[j];
            const char *src;
            if (head[j] < a.hq) {
                if (!APPEND && !a.Qo && place[tok[j]].win < 0) {  // only the window's queries are wanted
                    x[j] = (u32x4r){0u, 0u, 0u, 0u};
                    continue;
                }
                src = a.Q + ft * a.q_stride + (int64_t)head[j] * RB;
            } else if (head[j] < a.hq + a.hk) {
                src = a.K + ft * a.k_stride + (int64_t)(head[j] - a.hq) * RB;
            } else {
                src = a.V + ft * a.v_stride + (int64_t)(head[j] - a.hq - a.hk) * RB;
            }
            x[j] = *reinterpret_cast<const u32x4r *>(src + 16 * seg);
        }
#pragma unroll
        for (int j = 0; j < kRopeRows; ++j) {
            const bool live = r0 + j * RPI < rows;
            const bool isq = head[j] < a.hq, isv = head[j] >= a.hq + a.hk;
            float f[EL];
            unpack_row<BF>(x[j], f);
            if (a.qw || a.kw) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < EL; ++e) ss = fmaf(f[e], f[e], ss);
                const float inv = 1.f / sqrtf(row_sum<S>(ss) / (float)D + a.eps);  // (every lane takes part)
                if (isq ? a.qw != nullptr : a.kw != nullptr) {
#pragma unroll
                    for (int e = 0; e < EL; ++e) f[e] = f[e] * inv * wt[isq ? 0 : 1][e0 + e];
                }
            }
            if (a.rot > 0) {
                const float2 *c = cs[tok[j]];
                if (a.interleaved) {
                    if (e0 < a.rot) {
#pragma unroll
                        for (int e = 0; e < EL; e += 2) {
                            const float2 t = c[(e0 + e) >> 1];
                            const float u = f[e], v = f[e + 1];
                            f[e] = u * t.x - v * t.y;
                            f[e + 1] = v * t.x + u * t.y;
                        }
                    }
                } else {
                    const bool lo = e0 < half;
                    const int other = e0 >= a.rot ? (int)(threadIdx.x & 63)
                                                  : (int)(threadIdx.x & 63) + (lo ? half / EL : -(half / EL));
                    float g[EL];
#pragma unroll
                    for (int e = 0; e < EL; ++e) g[e] = __shfl(f[e], other, kWave);
                    if (e0 < a.rot) {
#pragma unroll
                        for (int e = 0; e < EL; ++e) {
                            const float2 t = c[(lo ? e0 : e0 - half) + e];
                            f[e] = lo ? f[e] * t.x - g[e] * t.y : f[e] * t.x + g[e] * t.y;
                        }
                    }
                }
            }
            const u32x4r y = isv ? x[j] : pack_row<BF>(f);
            if (!live) continue;
            const TokenPlace &p = place[tok[j]];
            const int64_t ft = first + tok[j];
            if (isq) {
                const int64_t row = APPEND ? ((int64_t)p.l * a.Hq + head[j]) * a.n + p.t : ft * a.Hq + head[j];
                if (a.Qo) *reinterpret_cast<u32x4r *>(a.Qo + row * RB + 16 * seg) = y;
                if (!APPEND && p.win >= 0)
                    *reinterpret_cast<u32x4r *>(a.win + (p.win + (int64_t)head[j] * a.B * a.w) * RB + 16 * seg) = y;
            } else if constexpr (APPEND) {
                const int h = head[j] - a.hq - (isv ? a.hk : 0);
                char *const out = isv ? a.Vo : a.Ko;
                if (p.tail >= 0)
                    *reinterpret_cast<u32x4r *>(out + (p.tail + ((int64_t)h << a.map.shift)) * RB + 16 * seg) = y;
            } else {
                *reinterpret_cast<u32x4r *>(a.Ko + (ft * a.Hkv + head[j] - a.hq) * RB + 16 * seg) = y;
            }
        }
    }
}

template <bool APPEND>
static void launch_rope(const RopeArgs &a, bool bf16, int D, dim3 grid, hipStream_t st)
{
    const dim3 b(kRopeThreads);
    if (bf16 && D == 128) hipLaunchKernelGGL((k_rope<true, 128, APPEND>), grid, b, 0, st, a);
    else if (bf16) hipLaunchKernelGGL((k_rope<true, 64, APPEND>), grid, b, 0, st, a);
    else if (D == 128) hipLaunchKernelGGL((k_rope<false, 128, APPEND>), grid, b, 0, st, a);
    else hipLaunchKernelGGL((k_rope<false, 64, APPEND>), grid, b, 0, st, a);
}

hipError_t rope_launch(RopeArgs a, bool append, bool bf16, int D, hipStream_t st)
{
    const int64_t all = (int64_t)a.L * a.n;
    a.per_block = all > 2 * kOneRound ? kRopeTokens : 1;
    const int64_t blocks = (all + a.per_block - 1) / a.per_block;
    const dim3 grid((unsigned)(blocks < kGridX ? blocks : kGridX), 1, (unsigned)((blocks + kGridX - 1) / kGridX));
    if (append) ECOKV_TIMED("append", st, (launch_rope<true>(a, bf16, D, grid, st)));
    else ECOKV_TIMED("prefill_rope", st, (launch_rope<false>(a, bf16, D, grid, st)));
    return hipGetLastError();
}

}  // namespace ecokv
