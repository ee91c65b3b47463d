// Rows that move inside the cache (gfx950): ecokv_commit, ecokv_evict and
// ecokv_evict_tails.
//
// Eviction in two launches.  k_evict_plan, a block per unit: the heaviest rows
// before the newest by a radix select on the masses' order-preserving keys, then, in
// the rows' order, the places that are free and the rows past the heavy ones' places
// that stay (the i-th of these goes to the i-th of those), and the masses at their
// new places.  k_evict_move: the rows themselves.  A row that stays where it is costs
// nothing, so a call moves the newest rows and at most as many others as were evicted.
#include "ecokv_internal.h"

namespace ecokv {

typedef unsigned int u32x4e __attribute__((ext_vector_type(4)));

// ---- commit ----

constexpr int kCommitThreads = 256;

// A block moves the K or the V rows of a (layer, KV head, continuation): all of them
// are in registers before the first is written, so their places may overlap.
template <int S>
__global__ __launch_bounds__(kCommitThreads) void k_commit(CommitArgs a)
{
    constexpr int EACH = 64 * S / kCommitThreads;  // 16-byte chunks of a thread at most
    const uint32_t b = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    const uint32_t u = b >> 1;
    if (u >= (uint32_t)a.units) return;
    const int lh = (int)(u / (uint32_t)a.N), c = (int)(u - (uint32_t)lh * (uint32_t)a.N);
    const int l = lh / a.Hkv, h = lh - l * a.Hkv;
    const int lane = threadIdx.x & 63;
    const int n = a.tail_counts[c], take = a.accepted[c];
    if (n < 0 || take <= 0 || take > a.nodes) return;
    // lane k: from where to where the k-th accepted row goes
    const int node = lane < take ? a.path[(int64_t)c * a.nodes + lane] : a.nodes + lane;
    const int before = __shfl_up(node, 1, kWave);
    const int from = (int)((uint32_t)n + (uint32_t)node), to = (int)((uint32_t)n + (uint32_t)lane);
    int pf = -1, pt = -1;
    bool good = lane >= take;
    if (!good) {
        pf = tail_page(a.map, c, from), pt = tail_page(a.map, c, to);
        good = node >= 0 && node < a.nodes && (lane == 0 || node > before) && pf >= 0 && pt >= 0;
    }
    if (__builtin_amdgcn_ballot_w64(good) != ~0ull) return;  // (the same in every wave)
    const int stay = __popcll(__builtin_amdgcn_ballot_w64(node == lane));  // (the first ones: the nodes ascend)
    char *const pool = b & 1 ? a.V : a.K;
    const int chunks = (take - stay) * S;
    u32x4e x[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = i * kCommitThreads + (int)threadIdx.x, k = min(stay + j / S, 63), seg = j % S;
        if (i * kCommitThreads < chunks) {
            const int r = __shfl(from, k, kWave), page = __shfl(pf, k, kWave);
            if (j < chunks) x[i] = *reinterpret_cast<const u32x4e *>(pool + tail_row(a.map, a.Hkv, l, h, page, r) * (16 * S) + 16 * seg);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = i * kCommitThreads + (int)threadIdx.x, k = min(stay + j / S, 63), seg = j % S;
        if (i * kCommitThreads < chunks) {
            const int r = __shfl(to, k, kWave), page = __shfl(pt, k, kWave);
            if (j < chunks) *reinterpret_cast<u32x4e *>(pool + tail_row(a.map, a.Hkv, l, h, page, r) * (16 * S) + 16 * seg) = x[i];
        }
    }
}

hipError_t commit_launch(const CommitArgs &a, hipStream_t st)
{
    const int64_t n = 2 * a.units;
    const dim3 g((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX)), b(kCommitThreads);
    if (a.row_bytes == 128) ECOKV_TIMED("commit", st, hipLaunchKernelGGL(k_commit<8>, g, b, 0, st, a));
    else if (a.row_bytes == 256) ECOKV_TIMED("commit", st, hipLaunchKernelGGL(k_commit<16>, g, b, 0, st, a));
    else ECOKV_TIMED("commit", st, hipLaunchKernelGGL(k_commit<32>, g, b, 0, st, a));
    return hipGetLastError();
}

// ---- eviction ----

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;
constexpr int kMoveThreads = 256;

// A unit: (layer, KV head) and group, a prompt of the compressed cache or a
// continuation with a tail; its row r is at `at`(r) of K, V and the masses.
struct EvictUnit {
    int lh, l, h, g;
    int64_t base;
};
__device__ __forceinline__ EvictUnit evict_unit(const EvictArgs &a, uint32_t u)
{
    EvictUnit x;
    x.lh = (int)(u / (uint32_t)a.groups);
    x.g = (int)(u - (uint32_t)x.lh * (uint32_t)a.groups);
    x.l = x.lh / a.Hkv;
    x.h = x.lh - x.l * a.Hkv;
    x.base = a.tails ? 0 : uniform_i32(a.offsets[u]);
    return x;
}
__device__ __forceinline__ int64_t evict_at(const EvictArgs &a, const EvictUnit &x, int r)
{
    if (!a.tails) return x.base + r;
    return tail_row(a.map, a.Hkv, x.l, x.h, max(tail_page(a.map, x.g, r), 0), r);
}

// Exclusive sums over the block of 0 or 1 of every thread; `total` of all.
__device__ __forceinline__ int block_rank(bool f, int *waves, int &total)
{
    const unsigned long long m = __builtin_amdgcn_ballot_w64(f);
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    __syncthreads();
    if (lane == 0) waves[wv] = __popcll(m);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kPlanWaves; ++i) {
        before += i < wv ? waves[i] : 0;
        total += waves[i];
    }
    return before + __popcll(m & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(kPlanThreads) void k_evict_plan(EvictArgs a)
{
    __shared__ uint32_t hist[2048];
    __shared__ int waves[kPlanWaves];
    __shared__ uint32_t pick[2];
    const uint32_t u = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    if (u >= (uint32_t)a.units) return;
    const int t = threadIdx.x;
    const EvictUnit x = evict_unit(a, u);
    const int n = uniform_i32(a.tails ? a.counts[x.g] : a.counts[u]);
    int *const head = a.plan + (int64_t)u * a.plan_stride;
    int *const src = head + kPlanHead, *const dst = src + a.cap;
    float *const mv = reinterpret_cast<float *>(dst + a.cap);
    bool out = n < 0 || n > a.max_rows;
    if (a.tails && !out) {
        int lost = 0;
        const int pages = (n + (1 << a.map.shift) - 1) >> a.map.shift;
        for (int p = t; p < pages; p += kPlanThreads) lost |= tail_page(a.map, x.g, p << a.map.shift) < 0;
        out = __syncthreads_or(lost);
    }
    if (t == 0) {
        head[0] = out || n <= a.limit ? -1 : 0;
        head[1] = n;
    }
    if (out) return;
    if (n <= a.limit) {  // nothing goes; another buffer gets the masses as they are
        if (a.mass_out != a.mass)
            for (int r = t; r < n; r += kPlanThreads) {
                const int64_t at = evict_at(a, x, r);
                a.mass_out[at] = a.mass[at];
            }
        return;
    }
    const int heavy = a.keep - a.recent, old = n - a.recent;
    // the key of the heavy-th heaviest of the older rows, digit by digit; `need` rows of it stay
    uint32_t key = 0, need = (uint32_t)heavy;
    if (heavy > 0) {
#pragma unroll 1
        for (int d = 0; d < 3; ++d) {
            const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bits = d == 2 ? 10 : 11;
            for (int i = t; i < 2048; i += kPlanThreads) hist[i] = 0;
            __syncthreads();
            for (int r = t; r < old; r += kPlanThreads) {
                const uint32_t q = score_key(a.mass[evict_at(a, x, r)]);
                if (d == 0 || (q >> (shift + bits)) == (key >> (shift + bits))) atomicAdd(&hist[(q >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // from the top: the first digit at which the rows so far reach `need`
            if (t < kWave) {
                const int per = (1 << bits) / kWave, top = (1 << bits) - 1 - t * per;
                uint32_t sum = 0;
                for (int i = 0; i < per; ++i) sum += hist[top - i];
                const uint32_t end = wave_incl_scan(sum);
                uint32_t left = need - (end - sum);
                if (end - sum < need && need <= end) {
                    int i = 0;
                    for (; hist[top - i] < left; ++i) left -= hist[top - i];
                    pick[0] = (uint32_t)(top - i);
                    pick[1] = left;
                }
            }
            __syncthreads();
            key |= pick[0] << shift;
            need = pick[1];
        }
    }
    // in the rows' order: which of them stay, the free places and the rows that fill them
    int equal = 0, holes = 0, movers = 0;
    for (int r0 = 0; r0 < old; r0 += kPlanThreads) {
        const int r = r0 + t;
        const float m = r < old ? a.mass[evict_at(a, x, r)] : 0.f;
        const uint32_t q = score_key(m);
        int total;
        const bool same = r < old && heavy > 0 && q == key;
        const int rank = equal + block_rank(same, waves, total);
        equal += total;
        const bool stays = r < old && heavy > 0 && (q > key || (same && (uint32_t)rank < need));
        const bool hole = r < heavy && !stays, mover = r >= heavy && stays;
        const int i = holes + block_rank(hole, waves, total);
        holes += total;
        const int j = movers + block_rank(mover, waves, total);
        movers += total;
        if (hole) dst[i] = r;
        if (mover) src[j] = r, mv[j] = m;
        if (stays && r < heavy && a.mass_out != a.mass) a.mass_out[evict_at(a, x, r)] = m;
    }
    __syncthreads();
    for (int i = t; i < movers; i += kPlanThreads) a.mass_out[evict_at(a, x, dst[i])] = mv[i];
    for (int r0 = 0; r0 < a.recent; r0 += kPlanThreads) {
        const int r = r0 + t;
        const float m = r < a.recent ? a.mass[evict_at(a, x, old + r)] : 0.f;
        __syncthreads();  // (a place may be a row that another thread has yet to read)
        if (r < a.recent) a.mass_out[evict_at(a, x, heavy + r)] = m;
    }
    if (t == 0) head[0] = movers;
}

// A block moves the chunks [c0, c0 + cols) of 16 bytes of a unit's rows, K's and V's
// side by side.
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a)
{
    const uint32_t b = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    const uint32_t u = b / (uint32_t)a.splits;
    if (u >= (uint32_t)a.units) return;
    const int split = (int)(b - u * (uint32_t)a.splits), t = threadIdx.x;
    const EvictUnit x = evict_unit(a, u);
    const int *const head = a.plan + (int64_t)u * a.plan_stride;
    const int *const src = head + kPlanHead, *const dst = src + a.cap;
    const int moves = uniform_i32(head[0]), n = uniform_i32(head[1]);
    if (split == 0 && t == 0) {
        if (!a.tails) a.new_counts[u] = moves < 0 ? n : a.keep;
        else if (x.lh == 0) a.new_counts[x.g] = moves < 0 ? n : a.keep;
    }
    if (moves < 0) return;
    const int cols = a.cols, per = kMoveThreads / cols;  // rows at a time
    const int chunk = split * cols + t % cols, S = a.row_bytes / 16, mine = t / cols;
    char *const pool = (chunk < S ? a.K : a.V) + 16 * (chunk % S);
    const auto row = [&](int r) { return reinterpret_cast<u32x4e *>(pool + evict_at(a, x, r) * a.row_bytes); };
    constexpr int U = 4;
    for (int i = 0; i < moves; i += U * per) {
        u32x4e v[U];
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = *row(src[min(i + j * per + mine, moves - 1)]);
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (i + j * per + mine < moves) *row(dst[i + j * per + mine]) = v[j];
    }
    __syncthreads();  // (a newest row's place may be one that moved from there)
    const int heavy = a.keep - a.recent, old = n - a.recent;
    for (int i = 0; i < a.recent; i += U * per) {
        u32x4e v[U];
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = *row(old + min(i + j * per + mine, a.recent - 1));
        __syncthreads();
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (i + j * per + mine < a.recent) *row(heavy + i + j * per + mine) = v[j];
    }
}

hipError_t evict_launch(EvictArgs a, hipStream_t st)
{
    const auto grid = [](int64_t n) {
        return dim3((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX));
    };
    ECOKV_TIMED("evict_plan", st, hipLaunchKernelGGL(k_evict_plan, grid(a.units), dim3(kPlanThreads), 0, st, a));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.cols = a.row_bytes / 16;
    a.splits = 2;
    ECOKV_TIMED("evict_move", st, hipLaunchKernelGGL(k_evict_move, grid(a.units * a.splits), dim3(kMoveThreads), 0, st, a));
    return hipGetLastError();
}

}  // namespace ecokv
