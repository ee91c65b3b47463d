// Norms and rotary positions (gfx950): ecokv_prefill_rope for a prompt's
// queries and keys, ecokv_append for the tokens that continue it.
//
// A row x [D] of a token at position p: x <- x / sqrt(mean x^2 + eps) w, then
// each pair (a, b) of rotated dimensions turns by p freq[i].  Every row is read
// and written once, so the calls are bound by HBM for prompts and by the
// latency of one launch for single tokens.
//
// A wave takes a token (or, in calls of few tokens, a quarter of its heads):
// positions, places and addresses are then scalars, and the cosines and sines,
// computed once per token, stay in registers for all its rows.  A load
// instruction covers 1024 consecutive bytes, a row the S = row bytes / 16 lanes
// of a group; the half-split layout's other dimension of a pair comes from the
// lane half a rotation away, the interleaved one's from the same lane.  A
// block's threads over the rows of four tokens, each finding its token and head
// and reading its cosines from LDS, were bound by vector instructions (us, before
// -> so: 32768 tokens of 28 + 4 heads of 128 bf16 elements 108 -> 96 = 5.6 TB/s,
// 15394 normed tokens of 32 + 8 heads 70 -> 60 = 5.3 TB/s, 2552 appended tokens
// 15.5 -> 13.1).
#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4r __attribute__((ext_vector_type(4)));

constexpr int kRopeThreads = 256, kRopeWaves = kRopeThreads / kWave;
constexpr int kRopeBatch = 4;  // rows a lane has in flight
// Tokens up to which a token's heads are dealt to a block's four waves (48 tokens
// of 32 + 8 + 8 heads 11.9 -> 8.2 us, their launch included).
constexpr int64_t kRopeSplit = 512;
// Bytes of a prompt's rows past which they go past the caches, whose 256 MB would
// not hold what was read and written until it is used again (268 MB 103 -> 96 us,
// 158 MB 68 -> 60).
constexpr int64_t kRopeStream = (int64_t)64 << 20;

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

// cos and sin of p w.  The angle is p w in turns, reduced to an eighth of one
// beside a quarter in 64 bits (the product of a 31-bit position and a 24-bit
// frequency needs more than 32 bits to keep its fraction; an eighth rounds to 32
// with 2.3e-8 radians at most, half a turn with 9.4e-8), the rest in 32.
__device__ __forceinline__ float2 turn(int p, float w, float factor)
{
    const double t = 4.0 * ((double)p * (double)w * 0.15915494309189533577), n = rint(t);
    const int q = (int)(n - 4.0 * floor(0.25 * n));  // quarters, 0 .. 3
    float s, c;
    sincospif(0.5f * (float)(t - n), &s, &c);
    const float cq = q & 1 ? -s : c, sq = q & 1 ? c : s;
    return q & 2 ? make_float2(-factor * cq, -factor * sq) : make_float2(factor * cq, factor * sq);
}

// The sequence of packed token t.
__device__ __forceinline__ int seq_of(const RopeArgs &a, int t)
{
    int s = 0;
    while (s + 1 < a.B && a.seq.cu[s + 1] <= t) ++s;
    return s;
}

// NT: rows are read and written past the caches.
template <bool BF, int D, bool APPEND, bool NORM, bool NT>
__global__ __launch_bounds__(kRopeThreads) void k_rope(RopeArgs a)
{
    constexpr int EL = BF ? 8 : 4;        // elements per lane
    constexpr int RB = D * (BF ? 2 : 4);  // row bytes
    constexpr int S = RB / 16;            // lanes per row
    constexpr int RPI = kWave / S;        // rows per load instruction
    constexpr int POLICY = NT ? 2 : 0;
    __shared__ __attribute__((aligned(16))) float2 cs[kRopeWaves][D / 2];
    const int lane = threadIdx.x & 63, wv = uniform_i32(threadIdx.x >> 6);
    const int64_t block = (int64_t)blockIdx.z * kGridX + blockIdx.x;
    // the wave's token, and which of its load instructions: w0, w0 + step, ...
    const int64_t ft = a.split ? block : block * kRopeWaves + wv;
    const int w0 = a.split ? wv : 0, step = a.split ? kRopeWaves : 1;
    if (ft >= (int64_t)a.L * a.n) return;
    const int l = (int)(ft / a.n), t = (int)(ft - (int64_t)l * a.n);
    const int seg = lane % S, e0 = seg * EL, half = a.rot >> 1;

    // a head's rows of the token as instructions nq, nk (and as many for V)
    const int nq = (a.hq + RPI - 1) / RPI, nk = (a.hk + RPI - 1) / RPI, all = nq + (APPEND ? 2 : 1) * nk;
    const auto rows = [&](const char *p, int64_t stride, int heads) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(uniform_ptr(p + ft * stride)), (short)0,
                                                 uniform_i32(heads * RB), 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t rq = rows(a.Q, a.q_stride, a.hq), rk = rows(a.K, a.k_stride, a.hk),
                                 rv = rows(a.V, a.v_stride, APPEND ? a.hk : 0);
    int64_t win = -1, tail = -1;  // prefill: row of Q_win of head 0; append: row of the tails of head 0
    const int pos = uniform_i32(APPEND || a.positions ? a.positions[t] : t - a.seq.cu[seq_of(a, t)]);
    if constexpr (APPEND) {
        const int row = uniform_i32(a.rows[t]), page = uniform_i32(tail_page(a.map, a.conts ? a.conts[t] : t, row));
        if (page >= 0) tail = tail_row(a.map, a.Hkv, l, 0, page, row);
    } else if (a.win) {
        const int s = seq_of(a, t), j = t - (a.seq.cu[s + 1] - a.w);
        if (j >= 0) win = ((int64_t)l * a.Hq * a.B + s) * a.w + j;
    }
    const bool want_q = APPEND || a.Qo || win >= 0;  // (else only the window's queries are wanted)

    u32x4r x[kRopeBatch];
    const auto load = [&](int i0) {  // instructions i0, i0 + step, ... (rows past a token's heads read zero)
#pragma unroll
        for (int j = 0; j < kRopeBatch; ++j) {
            const int i = i0 + j * step;
            if (i < nq) {
                if (want_q) x[j] = __builtin_bit_cast(u32x4r, __builtin_amdgcn_raw_buffer_load_b128(rq, i * 1024 + lane * 16, 0, POLICY));
            } else if (i < nq + nk) {
                x[j] = __builtin_bit_cast(u32x4r, __builtin_amdgcn_raw_buffer_load_b128(rk, (i - nq) * 1024 + lane * 16, 0, POLICY));
            } else if (APPEND && i < all) {
                x[j] = __builtin_bit_cast(u32x4r, __builtin_amdgcn_raw_buffer_load_b128(rv, (i - nq - nk) * 1024 + lane * 16, 0, POLICY));
            }
        }
    };
    load(w0);

    // A row's element e becomes  x[e] A[e] + h[e] B[e]  (times the norm's factor):
    // h is the pair's other element, A and B the cosine and sine times the norm's
    // weights of both, for queries and for keys (without norms alike).
    const bool turns = e0 < a.rot, lo = e0 < half;
    // the lane half a rotation away, whose element e pairs with this lane's
    const int other = turns && !a.interleaved ? lane + (lo ? half / EL : -(half / EL)) : lane;
    float A[NORM ? 2 : 1][EL], B[NORM ? 2 : 1][EL];
    {
        float c[EL], s[EL];
#pragma unroll
        for (int e = 0; e < EL; ++e) {
            c[e] = 1.f;
            s[e] = 0.f;
        }
        if (a.rot > 0) {
            if (lane < half) cs[wv][lane] = turn(pos, a.freq[lane], a.factor);
            // (a wave's own LDS accesses are ordered)
            if (turns) {
                const int p0 = a.interleaved ? e0 >> 1 : lo ? e0 : e0 - half;
#pragma unroll
                for (int e = 0; e < EL; ++e) {
                    const float2 v = cs[wv][a.interleaved ? p0 + (e >> 1) : p0 + e];
                    c[e] = v.x;
                    s[e] = (a.interleaved ? e & 1 : !lo) ? v.y : -v.y;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < (NORM ? 2 : 1); ++k) {
            float own[EL], far[EL];
#pragma unroll
            for (int e = 0; e < EL; ++e) own[e] = far[e] = 1.f;
            const char *w = static_cast<const char *>(k ? a.kw : a.qw);
            if (NORM && w) {
                unpack_row<BF>(*reinterpret_cast<const u32x4r *>(w + 16 * seg), own);
                unpack_row<BF>(*reinterpret_cast<const u32x4r *>(w + 16 * (seg + other - lane)), far);
            }
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                A[k][e] = own[e] * c[e];
                B[k][e] = (a.interleaved ? own[e ^ 1] : far[e]) * s[e];
            }
        }
    }

    for (int i0 = w0; i0 < all; i0 += kRopeBatch * step) {
        if (i0 != w0) load(i0);
#pragma unroll
        for (int j = 0; j < kRopeBatch; ++j) {
            const int i = i0 + j * step;
            if (i >= all || (i < nq && !want_q)) continue;
            const bool isq = i < nq, isv = APPEND && i >= nq + nk;
            u32x4r y = x[j];
            if (!isv) {
                float f[EL], h[EL];
                unpack_row<BF>(x[j], f);
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < EL; ++e) h[e] = turns ? f[e ^ 1] : 0.f;
                } else {
                    u32x4r z;
                    if (half == 8 * EL) {  // (eight lanes on: a move within 16 lanes)
#pragma unroll
                        for (int k = 0; k < 4; ++k) z[k] = dpp_u32<0x128>(x[j][k]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) z[k] = (unsigned)__shfl((int)x[j][k], other, kWave);
                    }
                    if (a.rot < D)  // (what stays is not added infinity times 0)
#pragma unroll
                        for (int k = 0; k < 4; ++k) z[k] = turns ? z[k] : 0u;
                    unpack_row<BF>(z, h);
                }
                float inv = 1.f;
                if constexpr (NORM) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < EL; ++e) ss = fmaf(f[e], f[e], ss);
                    ss = row_sum<S>(ss);
                    if (isq ? a.qw != nullptr : a.kw != nullptr) inv = __builtin_amdgcn_rsqf(ss * (1.f / D) + a.eps);
                }
                const int k = NORM && !isq ? 1 : 0;
#pragma unroll
                for (int e = 0; e < EL; ++e) f[e] = (f[e] * (k ? A[NORM][e] : A[0][e]) + h[e] * (k ? B[NORM][e] : B[0][e])) * inv;
                y = pack_row<BF>(f);
            }
            const int r = (isq ? i : isv ? i - nq - nk : i - nq) * RPI + lane / S;  // head
            if (r >= (isq ? a.hq : a.hk)) continue;
            if (isq) {
                if constexpr (APPEND) {
                    *reinterpret_cast<u32x4r *>(a.Qo + (((int64_t)l * a.Hq + r) * a.n + t) * RB + 16 * seg) = y;
                } else {
                    u32x4r *const q = reinterpret_cast<u32x4r *>(a.Qo + ft * a.Hq * RB + i * 1024 + lane * 16);
                    if (a.Qo) {
                        if constexpr (NT) __builtin_nontemporal_store(y, q);
                        else *q = y;
                    }
                    if (win >= 0) *reinterpret_cast<u32x4r *>(a.win + (win + (int64_t)r * a.B * a.w) * RB + 16 * seg) = y;
                }
            } else if constexpr (APPEND) {
                if (tail >= 0)
                    *reinterpret_cast<u32x4r *>((isv ? a.Vo : a.Ko) + (tail + ((int64_t)r << a.map.shift)) * RB + 16 * seg) = y;
            } else {
                u32x4r *const k = reinterpret_cast<u32x4r *>(a.Ko + ft * a.Hkv * RB + (i - nq) * 1024 + lane * 16);
                if constexpr (NT) __builtin_nontemporal_store(y, k);
                else *k = y;
            }
        }
    }
}

template <bool APPEND, bool NT>
static void launch_rope(const RopeArgs &a, bool bf16, int D, dim3 grid, hipStream_t st)
{
    const dim3 b(kRopeThreads);
    const bool norm = a.qw || a.kw;
    if (bf16 && D == 128) {
        if (norm) hipLaunchKernelGGL((k_rope<true, 128, APPEND, true, NT>), grid, b, 0, st, a);
        else hipLaunchKernelGGL((k_rope<true, 128, APPEND, false, NT>), grid, b, 0, st, a);
    } else if (bf16) {
        if (norm) hipLaunchKernelGGL((k_rope<true, 64, APPEND, true, NT>), grid, b, 0, st, a);
        else hipLaunchKernelGGL((k_rope<true, 64, APPEND, false, NT>), grid, b, 0, st, a);
    } else if (D == 128) {
        if (norm) hipLaunchKernelGGL((k_rope<false, 128, APPEND, true, NT>), grid, b, 0, st, a);
        else hipLaunchKernelGGL((k_rope<false, 128, APPEND, false, NT>), grid, b, 0, st, a);
    } else {
        if (norm) hipLaunchKernelGGL((k_rope<false, 64, APPEND, true, NT>), grid, b, 0, st, a);
        else hipLaunchKernelGGL((k_rope<false, 64, APPEND, false, NT>), grid, b, 0, st, a);
    }
}

hipError_t rope_launch(RopeArgs a, bool append, bool bf16, int D, hipStream_t st)
{
    const int64_t all = (int64_t)a.L * a.n;
    a.split = all <= kRopeSplit;
    const int64_t blocks = a.split ? all : (all + kRopeWaves - 1) / kRopeWaves;
    const dim3 grid((unsigned)(blocks < kGridX ? blocks : kGridX), 1, (unsigned)((blocks + kGridX - 1) / kGridX));
    const int64_t bytes = all * (a.hq + a.hk) * D * (bf16 ? 2 : 4);
    if (append) ECOKV_TIMED("append", st, (launch_rope<true, false>(a, bf16, D, grid, st)));
    else if (bytes > kRopeStream) ECOKV_TIMED("prefill_rope", st, (launch_rope<false, true>(a, bf16, D, grid, st)));
    else ECOKV_TIMED("prefill_rope", st, (launch_rope<false, false>(a, bf16, D, grid, st)));
    return hipGetLastError();
}

}  // namespace ecokv
