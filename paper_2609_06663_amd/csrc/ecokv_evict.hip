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

// A wave moves the rows of a (layer, KV head, continuation), as many at a time as its
// registers hold, all of these read before the first is written.  Most units have a few
// rows, so the time is a chain of four loads (accepted, path, page, row): a wave each and
// not a block lets more run at once (28 layers of 48 continuations, 15 rows each on
// average, us a call: a block for K and one for V 22.9, a wave each 20.2, a wave for both
// 19.0, rows stored past the L2 16.4, which is 77 MB at 4.6 TB/s).
template <int S>
__global__ __launch_bounds__(kCommitThreads) void k_commit(CommitArgs a)
{
    const uint32_t w = (blockIdx.z * (uint32_t)kGridX + blockIdx.x) * (kCommitThreads / kWave) + uniform_i32(threadIdx.x >> 6);
    const uint32_t u = w;
    if (u >= (uint32_t)a.units) return;
    const int lh = (int)(u / (uint32_t)a.N), c = (int)(u - (uint32_t)lh * (uint32_t)a.N);
    const int l = lh / a.Hkv, h = lh - l * a.Hkv;
    const int lane = threadIdx.x & 63;
    const int n = a.tail_counts[c], take = a.accepted[c];
    // lane k: from where to where the k-th accepted row goes
    const int path = a.path[(int64_t)c * a.nodes + min(lane, a.nodes - 1)];
    const bool tells = a.taken && lh == 0 && lane == 0;  // what every unit of the continuation finds
    if (n < 0 || take <= 0 || take > a.nodes) {
        if (tells) a.taken[c] = 0;
        return;
    }
    const int node = lane < take ? path : a.nodes + lane;
    const int before = __shfl_up(node, 1, kWave);
    const int from = (int)((uint32_t)n + (uint32_t)node), to = (int)((uint32_t)n + (uint32_t)lane);
    int pf = -1, pt = -1;
    bool good = lane >= take;
    if (!good) {
        pf = tail_page(a.map, c, from), pt = tail_page(a.map, c, to);
        good = node >= 0 && node < a.nodes && (lane == 0 || node > before) && pf >= 0 && pt >= 0;
    }
    const bool whole = __builtin_amdgcn_ballot_w64(good) == ~0ull;
    if (tells) a.taken[c] = whole ? take : 0;
    if (!whole) return;
    const int stay = __popcll(__builtin_amdgcn_ballot_w64(node == lane));  // (the first ones: the nodes ascend)
    const int chunks = (take - stay) * S;
    constexpr int AT = 8;  // loads of each in a row
    for (int i0 = 0; i0 < chunks; i0 += AT * kWave) {
        // (places are below the rows of later turns, which have yet to be read)
        u32x4e x[2][AT];
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            if (i0 + i * kWave >= chunks) break;
            const int j = min(i0 + i * kWave + lane, chunks - 1), k = stay + j / S;
            const int r = __shfl(from, k, kWave), page = __shfl(pf, k, kWave);
            const int64_t at = tail_row(a.map, a.Hkv, l, h, page, r) * (16 * S) + 16 * (j % S);
            x[0][i] = *reinterpret_cast<const u32x4e *>(a.K + at);
            x[1][i] = *reinterpret_cast<const u32x4e *>(a.V + at);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (a place may be another's row)
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            if (i0 + i * kWave >= chunks) break;
            const int j = i0 + i * kWave + lane, k = stay + min(j, chunks - 1) / S;
            const int r = __shfl(to, k, kWave), page = __shfl(pt, k, kWave);
            const int64_t at = tail_row(a.map, a.Hkv, l, h, page, r) * (16 * S) + 16 * (j % S);
            if (j < chunks) {
                __builtin_nontemporal_store(x[0][i], reinterpret_cast<u32x4e *>(a.K + at));
                __builtin_nontemporal_store(x[1][i], reinterpret_cast<u32x4e *>(a.V + at));
            }
        }
    }
}

hipError_t commit_launch(const CommitArgs &a, hipStream_t st)
{
    const int64_t n = (a.units + 3) / 4;  // blocks of four waves
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

// Set bits of a wave's mask below this lane's.
__device__ __forceinline__ int lanes_below(unsigned long long m)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
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
    return before + lanes_below(m);
}

// What a unit's block finds out before it selects: whether the unit is left alone, its
// rows, where its plan is.
struct EvictPlan {
    EvictUnit x;
    int n, heavy, old;
    int *head, *src, *dst;
};
__device__ __forceinline__ EvictPlan evict_plan(const EvictArgs &a, uint32_t u)
{
    EvictPlan p;
    p.x = evict_unit(a, u);
    p.n = uniform_i32(a.tails ? a.counts[p.x.g] : a.counts[u]);
    p.heavy = a.keep - a.recent;
    p.old = p.n - a.recent;
    p.head = a.plan + (int64_t)u * a.plan_stride;
    p.src = p.head + kPlanHead;
    p.dst = p.src + a.cap;
    return p;
}
// Whether this thread sees a row of the tail that has no page.
template <int T>
__device__ __forceinline__ int evict_lost(const EvictArgs &a, const EvictPlan &p)
{
    int lost = 0;
    if (a.tails) {
        const int pages = (p.n + (1 << a.map.shift) - 1) >> a.map.shift;
        for (int i = threadIdx.x; i < pages; i += T) lost |= tail_page(a.map, p.x.g, i << a.map.shift) < 0;
    }
    return lost;
}
// Not past the limit: nothing goes, another buffer gets the masses as they are.
template <int T>
__device__ __forceinline__ void evict_none(const EvictArgs &a, const EvictPlan &p)
{
    if (a.mass_out != a.mass)
        for (int r = threadIdx.x; r < p.n; r += T) {
            const int64_t at = evict_at(a, p.x, r);
            a.mass_out[at] = a.mass[at];
        }
}
// From the top digit of a histogram of 2048 down: the first at which the keys so far
// reach `need`; pick: that digit, and how many of its keys are needed.  All T threads.
template <int T>
__device__ __forceinline__ void pick_digit(const uint32_t *hist, uint32_t need, uint32_t *sums, uint32_t *pick)
{
    constexpr int EACH = 2048 / T, W = T / kWave;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6, low = (T - 1 - t) * EACH;
    uint32_t h[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) sum += h[i] = hist[low + i];
    uint32_t end = wave_incl_scan(sum);
    if (lane == 63) sums[wv] = end;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < W; ++i) end += i < wv ? sums[i] : 0;
    if (end - sum < need && need <= end) {
        uint32_t left = need - (end - sum);
        int d = 0;
#pragma unroll
        for (int i = EACH - 1; i >= 0; --i) {
            if (d == 0 && left <= h[i]) d = i + 1;
            left -= d == 0 ? h[i] : 0;
        }
        pick[0] = (uint32_t)(low + d - 1);
        pick[1] = left;
    }
    lds_barrier();
}

// A unit of at most T KPT rows: thread t has rows t, t + T, .., their keys in
// registers.  The key of the heavy-th heaviest row digit by digit (11, 11 and 10 bits)
// by histograms in LDS, until its digit has no more than kEvictFew keys: then one wave
// takes these and finds it bit by bit.  (By bits of all keys from the top, with the block
// counting for each of them, the selection took 11 and 12 of 31 and 22 us: 1792 units of
// 1152 rows, 160 of 5600.)
constexpr int kEvictFew = 256;
template <int T, int KPT>
__global__ __launch_bounds__(T) void k_evict_plan(EvictArgs a)
{
    constexpr int W = T / kWave, TAB = KPT * W;
    __shared__ __align__(16) uint32_t hist[2048];
    __shared__ uint32_t sums[W], pick[3], few[kEvictFew];
    __shared__ int tab[2][TAB];
    const uint32_t u = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    if (u >= (uint32_t)a.units) return;
    const int t = threadIdx.x, lane = t & 63, wv = uniform_i32(t >> 6);
    const EvictPlan p = evict_plan(a, u);
    const int n = p.n, heavy = p.heavy, old = p.old;
    if (t == 0) {
        p.head[0] = -1;
        p.head[1] = n;
    }
    if (n < 0 || n > a.max_rows) return;
    if (n <= a.limit) {
        if (__syncthreads_or(evict_lost<T>(a, p))) return;
        evict_none<T>(a, p);
        return;
    }
    uint32_t key[KPT];
    {
        int64_t at[KPT];
#pragma unroll
        for (int i = 0; i < KPT; ++i) at[i] = i * T < old ? evict_at(a, p.x, min(i * T + t, old - 1)) : 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) key[i] = i * T + t < old ? score_key(a.mass[at[i]]) : 0u;
    }
    for (int i = t; i < 2048; i += T) hist[i] = 0;
    if (t == 0) pick[2] = 0;
    if (__syncthreads_or(evict_lost<T>(a, p))) return;

    uint32_t least = 0, need = (uint32_t)heavy, equal = 0;  // the key, how many equal to it stay, how many there are
    if (heavy > 0) {
#pragma unroll 1
        for (int d = 0; d < 3; ++d) {
            const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bits = d == 2 ? 10 : 11;
            const auto among = [&](uint32_t k) { return d == 0 || (k >> (shift + bits)) == (least >> (shift + bits)); };
#pragma unroll
            for (int i = 0; i < KPT; ++i)
                if (i * T + t < old && among(key[i])) atomicAdd(&hist[(key[i] >> shift) & ((1u << bits) - 1)], 1u);
            __syncthreads();
            pick_digit<T>(hist, need, sums, pick);
            least |= pick[0] << shift;
            need = pick[1];
            const uint32_t many = hist[pick[0]];
            if (d == 2) {
                equal = many;
                break;
            }
            if (many <= (uint32_t)kEvictFew) {
                // those that share the digits so far
#pragma unroll
                for (int i = 0; i < KPT; ++i)
                    if (i * T + t < old && (key[i] >> shift) == (least >> shift)) few[atomicAdd(&pick[2], 1u)] = key[i];
                __syncthreads();
                if (wv == 0) {
                    uint32_t mine[kEvictFew / kWave], k = least;
#pragma unroll
                    for (int i = 0; i < kEvictFew / kWave; ++i) mine[i] = kWave * i + lane < (int)many ? few[kWave * i + lane] : 0u;
                    for (uint32_t bit = 1u << (shift - 1); bit; bit >>= 1) {
                        uint32_t c = 0;
#pragma unroll
                        for (int i = 0; i < kEvictFew / kWave; ++i) c += (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(mine[i] >= (k | bit)));
                        if (c >= need) k |= bit;
                    }
                    uint32_t above = 0, same = 0;
#pragma unroll
                    for (int i = 0; i < kEvictFew / kWave; ++i) {
                        above += (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(mine[i] > k));
                        same += (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(mine[i] == k && kWave * i + lane < (int)many));
                    }
                    if (lane == 0) pick[0] = k, pick[1] = need - above, pick[2] = same;
                }
                __syncthreads();
                least = pick[0];
                need = pick[1];
                equal = pick[2];
                break;
            }
            __syncthreads();  // (every thread has read hist)
            for (int i = t; i < 2048; i += T) hist[i] = 0;
            __syncthreads();
        }
    }

    // sums before each wave's 64 rows, of table k by wave k
    const auto before = [&](int tables) {
        lds_barrier();
        if (wv < tables) {
            int sum = 0;
            for (int b = 0; b < TAB; b += kWave) {
                const int v = b + lane < TAB ? tab[wv][b + lane] : 0;
                const int end = (int)wave_incl_scan((uint32_t)v);
                if (b + lane < TAB) tab[wv][b + lane] = sum + end - v;
                sum += __builtin_amdgcn_readlane(end, 63);
            }
            if (lane == 0) sums[wv] = (uint32_t)sum;
        }
        lds_barrier();
    };
    // Which rows stay: heavier ones, and of the equal ones the first `need` in the rows'
    // order.
    unsigned stays = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i)
        if (i * T < old) stays |= (unsigned)(i * T + t < old && heavy > 0 && key[i] >= least) << i;
    if (equal > need) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int c = __popcll(__builtin_amdgcn_ballot_w64((stays >> i) & (unsigned)(key[i] == least)));
            if (lane == 0) tab[0][i * W + wv] = c;
        }
        before(1);
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool s = (stays >> i) & (unsigned)(key[i] == least);
            if (s && (uint32_t)(tab[0][i * W + wv] + lanes_below(__builtin_amdgcn_ballot_w64(s))) >= need) stays &= ~(1u << i);
        }
        lds_barrier();  // (tab is free again)
    }
    // the places that are free (rows below `heavy` that go), and the rows that fill them
    // (from there on that stay)
    const auto lows = [&](int i) {
        const int d = heavy - (i * T + wv * kWave);
        return d >= 64 ? ~0ull : d > 0 ? (1ull << d) - 1 : 0ull;
    };
    unsigned long long odd[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        odd[i] = i * T < old ? __builtin_amdgcn_ballot_w64((stays >> i) & 1u) ^ lows(i) : 0;
        if (lane == 0) tab[0][i * W + wv] = __popcll(odd[i] & lows(i)), tab[1][i * W + wv] = __popcll(odd[i] & ~lows(i));
    }
    before(2);
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        if (i * T >= old) continue;
        const bool low = i * T + t < heavy;
        if (!((odd[i] >> lane) & 1)) continue;
        const int at = tab[low ? 0 : 1][i * W + wv] + lanes_below(odd[i] & (low ? lows(i) : ~lows(i)));
        (low ? p.dst : p.src)[at] = i * T + t;
    }
    if (t == 0) p.head[0] = (int)sums[1];
}

// The same for units of any number of rows, whose masses are read again for every
// digit of the key.
__global__ __launch_bounds__(kPlanThreads) void k_evict_plan_long(EvictArgs a)
{
    __shared__ uint32_t hist[2048];
    __shared__ int waves[kPlanWaves];
    __shared__ uint32_t pick[2];
    const uint32_t u = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    if (u >= (uint32_t)a.units) return;
    const int t = threadIdx.x;
    const EvictPlan p = evict_plan(a, u);
    const EvictUnit &x = p.x;
    const int n = p.n, heavy = p.heavy, old = p.old;
    if (t == 0) {
        p.head[0] = -1;
        p.head[1] = n;
    }
    if (n < 0 || n > a.max_rows || __syncthreads_or(evict_lost<kPlanThreads>(a, p))) return;
    if (n <= a.limit) {
        evict_none<kPlanThreads>(a, p);
        return;
    }
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
        const uint32_t q = score_key(r < old ? a.mass[evict_at(a, x, r)] : 0.f);
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
        if (hole) p.dst[i] = r;
        if (mover) p.src[j] = r;
    }
    if (t == 0) p.head[0] = movers;
}

// The masses of a unit's rows to their new places, in the order of the rows' moves.
__device__ __forceinline__ void move_masses(const EvictArgs &a, const EvictUnit &x, const int *src, const int *dst, int moves, int n)
{
    const int t = threadIdx.x, heavy = a.keep - a.recent, old = n - a.recent;
    if (a.mass_out != a.mass) {  // (what goes too; its places are filled after)
        for (int r = t; r < heavy; r += kMoveThreads) {
            const int64_t at = evict_at(a, x, r);
            a.mass_out[at] = a.mass[at];
        }
        __syncthreads();
    }
    for (int i = t; i < moves; i += kMoveThreads) a.mass_out[evict_at(a, x, dst[i])] = a.mass[evict_at(a, x, src[i])];
    __syncthreads();
    for (int r0 = 0; r0 < a.recent; r0 += kMoveThreads) {
        const int r = r0 + t;
        const float m = r < a.recent ? a.mass[evict_at(a, x, old + r)] : 0.f;
        __syncthreads();  // (a place may be a row that another thread has yet to read)
        if (r < a.recent) a.mass_out[evict_at(a, x, heavy + r)] = m;
    }
    // (a tail grows again: a row that comes to such a place begins with nothing)
    if (a.tails && a.mass_out == a.mass)
        for (int r = a.keep + t; r < n; r += kMoveThreads) a.mass_out[evict_at(a, x, r)] = 0.f;
}

// A block moves the chunks [c0, c0 + cols) of 16 bytes of a unit's rows, K's and V's
// side by side; one more block per unit the masses.  Rows are stored past the L2, which
// their loads then have to themselves (us a call, 28 layers of 16 tails of 1152 rows 121
// and 114, 160 units of 6553 rows 63.5 and 56.2; loads past it as well: 110 and 60.3).
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a)
{
    const uint32_t b = blockIdx.z * (uint32_t)kGridX + blockIdx.x;
    // (the masses' blocks come last: in between they would leave the rows' to half of the
    // XCDs, 134 us instead of 80)
    const uint32_t rows = (uint32_t)(a.units * a.splits);
    const bool masses = b >= rows;
    const uint32_t u = masses ? b - rows : b / (uint32_t)a.splits;
    if (u >= (uint32_t)a.units) return;
    const int split = (int)(b - u * (uint32_t)a.splits), t = threadIdx.x;
    const EvictUnit x = evict_unit(a, u);
    const int *const head = a.plan + (int64_t)u * a.plan_stride;
    const int *const src = head + kPlanHead, *const dst = src + a.cap;
    const int moves = uniform_i32(head[0]), n = uniform_i32(head[1]);
    if (masses && t == 0) {
        if (!a.tails) a.new_counts[u] = moves < 0 ? n : a.keep;
        else if (x.lh == 0) a.new_counts[x.g] = moves < 0 ? n : a.keep;
    }
    if (moves < 0) return;
    if (masses) {
        move_masses(a, x, src, dst, moves, n);
        return;
    }
    const int cols = a.cols, per = kMoveThreads / cols;  // rows at a time
    const int chunk = split * cols + t % cols, S = a.row_bytes / 16, mine = t / cols;
    char *const pool = (chunk < S ? a.K : a.V) + 16 * (chunk % S);
    const auto row = [&](int r) { return reinterpret_cast<u32x4e *>(pool + evict_at(a, x, r) * a.row_bytes); };
    constexpr int U = 4;
    const int step = U * per;
    u32x4e v[U], w[U];
    // the rows that fill free places; their numbers are read a step ahead
    const auto number = [&](const int *list, int i, int (&r)[U]) {
#pragma unroll
        for (int j = 0; j < U; ++j) r[j] = list[max(min(i + j * per + mine, moves - 1), 0)];
    };
    int from[U], to[U], from2[U], to2[U];
    if (moves > 0) number(src, 0, from), number(dst, 0, to);
    for (int i = 0; i < moves; i += step) {
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = *row(from[j]);
        number(src, i + step, from2), number(dst, i + step, to2);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i + j * per + mine < moves) __builtin_nontemporal_store(v[j], row(to[j]));
            from[j] = from2[j], to[j] = to2[j];
        }
    }
    __syncthreads();  // (a newest row's place may be one that moved from there)
    // The newest rows, a step's loads ahead of the stores of the one before: a place is
    // below every row of the steps after, and where it may be a row of its own step the
    // block waits for that step's loads.
    const int heavy = a.keep - a.recent, old = n - a.recent;
    const bool apart = n - a.keep >= a.recent;
    const auto load = [&](u32x4e (&x)[U], int i) {
#pragma unroll
        for (int j = 0; j < U; ++j) x[j] = *row(old + max(min(i + j * per + mine, a.recent - 1), 0));
    };
    if (a.recent > 0) load(v, 0);
    for (int i = 0; i < a.recent; i += step) {
        if (!apart) {
#pragma unroll
            for (int j = 0; j < U; ++j) asm volatile("" ::"v"(v[j]));  // (loaded)
            lds_barrier();
        }
        if (i + step < a.recent) load(w, i + step);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i + j * per + mine < a.recent) __builtin_nontemporal_store(v[j], row(heavy + i + j * per + mine));
            v[j] = w[j];
        }
    }
}

hipError_t evict_launch(EvictArgs a, hipStream_t st)
{
    const auto grid = [](int64_t n) {
        return dim3((unsigned)(n < kGridX ? n : kGridX), 1, (unsigned)((n + kGridX - 1) / kGridX));
    };
    const dim3 units = grid(a.units);
    // A unit's keys stay in registers where they fit, 8 a thread, in the fewest threads: a
    // rule on the bound, as the counts are the device's.  Past 8192 rows the masses are read
    // again for each digit, also of units that have fewer.  (us a plan: 28 layers of 4 heads
    // and 16 tails of 1152 rows, 256 and 1024 threads, 20.2 59.4; 4 units of 2048 rows 9.4
    // 10.0; 4 units of 8192 rows under bounds of 8192 and 8193 13.7 25.3, 160 of up to 6553
    // under 6553 and 26212 13.8 22.8; 4 of 16384 rows 42.1, of 26212 62.8.)
    if (a.max_rows <= 2048) ECOKV_TIMED("evict_plan", st, hipLaunchKernelGGL((k_evict_plan<256, 8>), units, dim3(256), 0, st, a));
    else if (a.max_rows <= 8192) ECOKV_TIMED("evict_plan", st, hipLaunchKernelGGL((k_evict_plan<1024, 8>), units, dim3(1024), 0, st, a));
    else ECOKV_TIMED("evict_plan", st, hipLaunchKernelGGL(k_evict_plan_long, units, dim3(kPlanThreads), 0, st, a));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // chunks of a row's K and V that a block moves: all of them, or fewer where that
    // leaves fewer than four blocks for each compute unit, down to 128 bytes
    a.cols = a.row_bytes / 8;
    while (a.cols > 8 && a.units * (a.row_bytes / 8 / a.cols) < 4 * kShBlocks) a.cols /= 2;
    a.splits = a.row_bytes / 8 / a.cols;
    ECOKV_TIMED("evict_move", st, hipLaunchKernelGGL(k_evict_move, grid(a.units * (a.splits + 1)), dim3(kMoveThreads), 0, st, a));
    return hipGetLastError();
}

}  // namespace ecokv
