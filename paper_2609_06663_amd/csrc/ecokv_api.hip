// C entry points of libecokv: host-side argument checks, workspace layout and
// launches.  Every check completes before anything is enqueued.
#include <math.h>
#include <stdlib.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <mutex>
#include <vector>

#include "ecokv_internal.h"

namespace {

thread_local char g_err[512] = "";

int fail(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return code;
}

struct ShapeInfo {
    int L, Hq, Hkv, G, D, w, B, R;
    int64_t Ttot, Ptot;
    int maxT, maxP;
};

// The layers, heads and head_dim of a shape.
int check_heads(const ecokv_shape *sh, ShapeInfo *o)
{
    if (!sh) return fail(ECOKV_EINVAL, "shape is NULL");
    if (sh->num_layers < 0) return fail(ECOKV_EINVAL, "num_layers %d < 0", sh->num_layers);
    if (sh->num_kv_heads < 1) return fail(ECOKV_EINVAL, "num_kv_heads %d < 1", sh->num_kv_heads);
    if (sh->num_q_heads < sh->num_kv_heads || sh->num_q_heads % sh->num_kv_heads != 0)
        return fail(ECOKV_EINVAL, "num_q_heads %d is not a positive multiple of num_kv_heads %d", sh->num_q_heads,
                    sh->num_kv_heads);
    if (sh->head_dim != 64 && sh->head_dim != 128)
        return fail(ECOKV_EUNSUPPORTED, "head_dim %d (supported: 64, 128)", sh->head_dim);
    o->L = sh->num_layers;
    o->Hq = sh->num_q_heads;
    o->Hkv = sh->num_kv_heads;
    o->G = o->Hq / o->Hkv;
    o->D = sh->head_dim;
    return ECOKV_OK;
}

// And its sequences, of more than `shortest` tokens.
int check_seqs(const ecokv_shape *sh, int shortest, ShapeInfo *o)
{
    if (sh->num_seqs < 1 || sh->num_seqs > ECOKV_MAX_SEQS)
        return fail(ECOKV_EINVAL, "num_seqs %d outside [1, %d]", sh->num_seqs, ECOKV_MAX_SEQS);
    if (!sh->cu_seqlens) return fail(ECOKV_EINVAL, "cu_seqlens is NULL");
    if (sh->cu_seqlens[0] != 0) return fail(ECOKV_EINVAL, "cu_seqlens[0] = %d, must be 0", sh->cu_seqlens[0]);
    o->maxT = 0;
    for (int s = 0; s < sh->num_seqs; ++s) {
        const int64_t T = (int64_t)sh->cu_seqlens[s + 1] - sh->cu_seqlens[s];
        if (T <= shortest && shortest > 0)
            return fail(ECOKV_EINVAL, "sequence %d has %lld tokens; the window %d must be shorter", s, (long long)T,
                        shortest);
        if (T <= shortest) return fail(ECOKV_EINVAL, "sequence %d has %lld tokens", s, (long long)T);
        if (T > o->maxT) o->maxT = (int)T;
    }
    o->B = sh->num_seqs;
    o->Ttot = sh->cu_seqlens[o->B];
    return ECOKV_OK;
}

int check_shape(const ecokv_shape *sh, ShapeInfo *o)
{
    int rc = check_heads(sh, o);
    if (rc) return rc;
    if (sh->window < 1) return fail(ECOKV_EINVAL, "window %d < 1", sh->window);
    if ((rc = check_seqs(sh, sh->window, o))) return rc;
    o->w = sh->window;
    o->R = o->G * o->w;
    o->Ptot = o->Ttot - (int64_t)o->B * o->w;
    o->maxP = o->maxT - o->w;
    if ((int64_t)o->L * o->Hkv * o->B > (int64_t)INT32_MAX / 8)
        return fail(ECOKV_EINVAL, "too many (layer, head, sequence) units");
    return ECOKV_OK;
}

int check_params(const ecokv_params *p)
{
    if (!p) return fail(ECOKV_EINVAL, "params is NULL");
    if (!(isfinite(p->alpha) && isfinite(p->beta) && isfinite(p->eps) && isfinite(p->tau)))
        return fail(ECOKV_EINVAL, "alpha, beta, eps and tau must be finite");
    if (p->eps < 0.f) return fail(ECOKV_EINVAL, "eps %g < 0", (double)p->eps);
    if (p->pool_kernel < 1 || p->pool_kernel % 2 == 0)
        return fail(ECOKV_EINVAL, "pool_kernel %d must be odd and >= 1", p->pool_kernel);
    if (p->causal != 0 && p->causal != 1) return fail(ECOKV_EINVAL, "causal must be 0 or 1");
    if (isinf(p->lambda_override)) return fail(ECOKV_EINVAL, "lambda_override must be NaN or finite");
    if (p->imp_mode != ECOKV_IMP_ATTN && p->imp_mode != ECOKV_IMP_ATTN_VNORM)
        return fail(ECOKV_EINVAL, "imp_mode %d", p->imp_mode);
    if (p->norm_mode < ECOKV_NORM_MINMAX || p->norm_mode > ECOKV_NORM_MAD)
        return fail(ECOKV_EINVAL, "norm_mode %d", p->norm_mode);
    if (!(p->winsor_q >= 0.f && p->winsor_q < 0.5f))
        return fail(ECOKV_EINVAL, "winsor_q %g outside [0, 0.5)", (double)p->winsor_q);
    if (!(isfinite(p->mad_tau) && p->mad_tau > 0.f)) return fail(ECOKV_EINVAL, "mad_tau %g", (double)p->mad_tau);
    if (p->redundancy != ECOKV_RED_EUCLID && p->redundancy != ECOKV_RED_STD)
        return fail(ECOKV_EINVAL, "redundancy %d", p->redundancy);
    if (p->centroid_scope != ECOKV_CENTROID_ALL && p->centroid_scope != ECOKV_CENTROID_PREFIX)
        return fail(ECOKV_EINVAL, "centroid_scope %d", p->centroid_scope);
    return ECOKV_OK;
}

int fill_seqtab(const ecokv_shape *sh, const int32_t *budget, int w, ecokv::SeqTab *t, int64_t *per_lh)
{
    memset(t, 0, sizeof *t);
    t->nseq = sh->num_seqs;
    for (int s = 0; s <= sh->num_seqs; ++s) t->cu[s] = sh->cu_seqlens[s];
    int64_t acc = 0;
    t->boff[0] = 0;
    for (int s = 0; s < sh->num_seqs; ++s) {
        const int T = sh->cu_seqlens[s + 1] - sh->cu_seqlens[s];
        int b = T;
        if (budget) {
            if (budget[s] < w)
                return fail(ECOKV_EINVAL, "budget[%d] = %d is below the window %d", s, budget[s], w);
            b = budget[s] < T ? budget[s] : T;
        }
        t->beff[s] = b;
        acc += b;
        if (acc > INT32_MAX) return fail(ECOKV_EINVAL, "budget sum overflows");
        t->boff[s + 1] = (int)acc;
    }
    if (per_lh) *per_lh = acc;
    return ECOKV_OK;
}

// Per-(layer, KV head) budgets (ECOKV_HEAD_BUDGETS): checks every budget and
// counts the idx entries, sum over (l, h, s) of min(b^l_h, T_s).
int head_budget_total(const ecokv_shape *sh, const ShapeInfo &si, const int32_t *budget, int64_t *total)
{
    const int64_t n = (int64_t)si.L * si.Hkv;
    int64_t acc = 0;
    for (int64_t j = 0; j < n; ++j) {
        if (budget[j] < si.w)
            return fail(ECOKV_EINVAL, "budget[%lld] = %d is below the window %d", (long long)j, budget[j], si.w);
        for (int s = 0; s < si.B; ++s) {
            const int T = sh->cu_seqlens[s + 1] - sh->cu_seqlens[s];
            acc += budget[j] < T ? budget[j] : T;
        }
        if (acc > INT32_MAX) return fail(ECOKV_EINVAL, "index count overflows int32");
    }
    *total = acc;
    return ECOKV_OK;
}

// The table of pairs lh0 .. lh0+n-1 (n <= kLhChunk) whose entries start at
// idx offset e0; returns the offset just past them.
int64_t fill_lhtab(const ecokv_shape *sh, int B, const int32_t *budget, int64_t lh0, int n, int64_t e0,
                   ecokv::LhTab *t)
{
    t->lh0 = (int)lh0;
    t->n = n;
    int64_t e = e0;
    for (int j = 0; j < n; ++j) {
        const int b = budget[lh0 + j];
        t->b[j] = b;
        t->start[j] = (int)e;
        for (int s = 0; s < B; ++s) {
            const int T = sh->cu_seqlens[s + 1] - sh->cu_seqlens[s];
            e += b < T ? b : T;
        }
    }
    t->start[n] = (int)e;
    return e;
}

int hip_fail(hipError_t e, const char *what)
{
    return fail(ECOKV_EHIP, "%s: %s", what, hipGetErrorString(e));
}

struct StageRec {
    const char *name;
    hipEvent_t start, stop;
};
std::mutex g_stage_mu;
std::vector<StageRec> g_stages;
thread_local const char *g_stage_name = nullptr;
thread_local hipEvent_t g_stage_start = nullptr;

// Groups of the largest select launch and keys of the largest group, which
// size the select workspace.
void select_dims(const ShapeInfo &si, const ecokv_shape *sh, int mode, int64_t *groups, int64_t *maxn)
{
    const int64_t pairs = (int64_t)si.L * si.Hkv;
    *groups = mode == ECOKV_HEAD_BUDGETS ? (pairs < ecokv::kLhChunk ? pairs : ecokv::kLhChunk) * si.B
              : mode == ECOKV_LAYER_FLAT ? (int64_t)si.L * si.B
                                         : pairs * si.B;
    *maxn = (int64_t)si.maxP * (mode == ECOKV_LAYER_FLAT ? si.Hkv : 1);
    (void)sh;
}

int check_select_mode(const ShapeInfo &si, int mode)
{
    if (mode != ECOKV_PER_HEAD && mode != ECOKV_LAYER_FLAT && mode != ECOKV_HEAD_BUDGETS)
        return fail(ECOKV_EINVAL, "mode %d", mode);
    if (mode == ECOKV_LAYER_FLAT) {
        if (si.Hkv > ecokv::select_max_flat_heads())
            return fail(ECOKV_EUNSUPPORTED, "LAYER_FLAT supports at most %d KV heads", ecokv::select_max_flat_heads());
        // (a selection group's scores are read through one 32-bit-addressed buffer descriptor)
        if ((int64_t)si.Hkv * si.Ptot * 4 > INT32_MAX)
            return fail(ECOKV_EUNSUPPORTED, "LAYER_FLAT: H_kv x P_total scores of a layer exceed 2^31 bytes");
    }
    if ((int64_t)si.maxP * 4 > INT32_MAX)
        return fail(ECOKV_EUNSUPPORTED, "a sequence's scores exceed 2^31 bytes");
    return ECOKV_OK;
}

// Checks the caller's select workspace and points the launch at it.
int select_workspace(const ShapeInfo &si, const ecokv_shape *shape, int mode, void *workspace, size_t workspace_bytes,
                     ecokv::SelectArgs *a)
{
    int64_t groups = 0, maxn = 0;
    select_dims(si, shape, mode, &groups, &maxn);
    const size_t need = ecokv::select_ws_layout(groups, maxn, mode != ECOKV_LAYER_FLAT).total;
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need)
        return fail(ECOKV_EWORKSPACE, "select workspace has %zu bytes, needs %zu", workspace_bytes, need);
    a->mb_groups = groups;
    a->mb_maxn = maxn;
    a->ws_bytes = workspace_bytes;
    return ECOKV_OK;
}

int score_impl(const void *K, const void *V, const void *Q_win, int dtype, const ecokv_shape *shape,
               const ecokv_params *params, const float *pre, float *scores, float *lambda, float *stats,
               void *workspace, size_t workspace_bytes, void *stream, bool noalloc);

// Scratch of ecokv_score_noalloc: a file-scope device array, one copy on
// every device the library runs on, kept until the process ends.  In host
// code `scratch` names a host-side stand-in, not device memory: its device
// address comes from hipGetSymbolAddress, taken once per device (with that
// device current) on the entry point's first call there and kept here.
constexpr size_t kNoAllocBytes = (size_t)96 << 20;
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void *g_scratch[kMaxDevices];

}  // namespace

static __device__ __align__(256) unsigned char scratch[kNoAllocBytes];

namespace {

// The scratch's device address on the current device, which must be the
// stream's device.
int noalloc_scratch(hipStream_t stream, void **out)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "ecokv_score_noalloc: hipGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return fail(ECOKV_EUNSUPPORTED, "ecokv_score_noalloc: device %d", dev);
    if (stream) {
        hipDevice_t sdev = -1;
        if ((e = hipStreamGetDevice(stream, &sdev)) != hipSuccess)
            return hip_fail(e, "ecokv_score_noalloc: hipStreamGetDevice");
        if ((int)sdev != dev)
            return fail(ECOKV_EINVAL, "ecokv_score_noalloc: the stream belongs to device %d, device %d is current",
                        (int)sdev, dev);
    }
    std::lock_guard<std::mutex> lk(g_scratch_mu);
    if (!g_scratch[dev]) {
        void *p = nullptr;
        if ((e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch))) != hipSuccess)
            return hip_fail(e, "ecokv_score_noalloc: hipGetSymbolAddress");
        if (!p || ((uintptr_t)p & 255u) != 0) return fail(ECOKV_EHIP, "ecokv_score_noalloc: bad scratch address");
        g_scratch[dev] = p;
    }
    *out = g_scratch[dev];
    return ECOKV_OK;
}

}  // namespace

namespace ecokv {

bool stage_timing_on()
{
    const char *v = getenv("ECOKV_STAGE_TIMING");
    return v && v[0] == '1' && v[1] == 0;
}

void stage_begin(const char *name, hipStream_t st)
{
    g_stage_name = nullptr;
    if (!stage_timing_on()) return;
    if (hipEventCreate(&g_stage_start) != hipSuccess) return;
    if (hipEventRecord(g_stage_start, st) != hipSuccess) {
        (void)hipEventDestroy(g_stage_start);
        return;
    }
    g_stage_name = name;
}

void stage_end(hipStream_t st)
{
    if (!g_stage_name) return;
    hipEvent_t stop;
    if (hipEventCreate(&stop) != hipSuccess || hipEventRecord(stop, st) != hipSuccess) {
        (void)hipEventDestroy(g_stage_start);
        g_stage_name = nullptr;
        return;
    }
    std::lock_guard<std::mutex> lk(g_stage_mu);
    g_stages.push_back({g_stage_name, g_stage_start, stop});
    g_stage_name = nullptr;
}

}  // namespace ecokv

extern "C" {

int ecokv_stage_times(ecokv_stage_time *out, int max, int *count)
{
    if (!count || (max > 0 && !out) || max < 0) return fail(ECOKV_EINVAL, "ecokv_stage_times: bad arguments");
    std::vector<StageRec> recs;
    {
        std::lock_guard<std::mutex> lk(g_stage_mu);
        recs.swap(g_stages);
    }
    int n = 0, rc = ECOKV_OK;
    for (const StageRec &r : recs) {
        float ms = 0.f;
        hipError_t e = hipEventSynchronize(r.stop);
        if (e == hipSuccess) e = hipEventElapsedTime(&ms, r.start, r.stop);
        (void)hipEventDestroy(r.start);
        (void)hipEventDestroy(r.stop);
        if (e != hipSuccess) {
            rc = hip_fail(e, "ecokv_stage_times");
            continue;
        }
        int k = 0;
        while (k < n && strcmp(out[k].name, r.name) != 0) ++k;
        if (k == n) {
            if (n >= max) continue;
            memset(&out[n], 0, sizeof out[n]);
            strncpy(out[n].name, r.name, sizeof out[n].name - 1);
            ++n;
        }
        out[k].ms += ms;
        out[k].launches += 1;
    }
    *count = n;
    return rc;
}


int ecokv_default_params(ecokv_params *p)
{
    if (!p) return fail(ECOKV_EINVAL, "params is NULL");
    p->alpha = 0.8f;
    p->beta = 0.6f;
    p->eps = 1e-6f;
    p->tau = 0.f;
    p->pool_kernel = 5;
    p->causal = 1;
    p->lambda_override = NAN;
    p->imp_mode = ECOKV_IMP_ATTN;
    p->norm_mode = ECOKV_NORM_MINMAX;
    p->winsor_q = 0.01f;
    p->mad_tau = 1.f;
    p->redundancy = ECOKV_RED_EUCLID;
    p->centroid_scope = ECOKV_CENTROID_ALL;
    return ECOKV_OK;
}

int ecokv_workspace_size(const ecokv_shape *shape, const ecokv_params *params, size_t *bytes)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_params(params))) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    if (si.R > ECOKV_MAX_ROWS)
        return fail(ECOKV_EUNSUPPORTED, "(H_q/H_kv)*window = %d exceeds %d", si.R, ECOKV_MAX_ROWS);
    *bytes = 0;  // the size depends on the element type; report the larger layout
    {
        const bool vn = params->imp_mode == ECOKV_IMP_ATTN_VNORM;
        const size_t b0 = ecokv::score_ws_layout(si.L, si.Hkv, si.B, si.D, si.R, si.Ptot, si.maxT, true, vn).total;
        const size_t b1 = ecokv::score_ws_layout(si.L, si.Hkv, si.B, si.D, si.R, si.Ptot, si.maxT, false, vn).total;
        *bytes = b0 > b1 ? b0 : b1;
    }
    return ECOKV_OK;
}

int ecokv_score(const void *K, const void *Q_win, int dtype, const ecokv_shape *shape, const ecokv_params *params,
                float *scores, float *lambda, float *stats, void *workspace, size_t workspace_bytes, void *stream)
{
    if (params && params->imp_mode != ECOKV_IMP_ATTN)
        return fail(ECOKV_EINVAL, "imp_mode %d needs the values: use ecokv_score_v", params->imp_mode);
    return ecokv_score_v(K, nullptr, Q_win, dtype, shape, params, scores, lambda, stats, workspace,
                         workspace_bytes, stream);
}

int ecokv_score_v(const void *K, const void *V, const void *Q_win, int dtype, const ecokv_shape *shape,
                  const ecokv_params *params, float *scores, float *lambda, float *stats, void *workspace,
                  size_t workspace_bytes, void *stream)
{
    return ecokv_score_pre(K, V, Q_win, dtype, shape, params, nullptr, scores, lambda, stats, workspace,
                           workspace_bytes, stream);
}

int ecokv_score_pre(const void *K, const void *V, const void *Q_win, int dtype, const ecokv_shape *shape,
                    const ecokv_params *params, const float *pre, float *scores, float *lambda, float *stats,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    return score_impl(K, V, Q_win, dtype, shape, params, pre, scores, lambda, stats, workspace, workspace_bytes,
                      stream, false);
}

int ecokv_score_noalloc(const void *K, const void *V, const void *Q_win, int dtype, const ecokv_shape *shape,
                        const ecokv_params *params, const float *pre, float *scores, float *lambda, float *stats,
                        void *stream)
{
    void *ws = nullptr;
    const int rc = noalloc_scratch(static_cast<hipStream_t>(stream), &ws);
    if (rc) return rc;
    return score_impl(K, V, Q_win, dtype, shape, params, pre, scores, lambda, stats, ws, kNoAllocBytes, stream,
                      true);
}

}  // extern "C"

namespace {

int score_impl(const void *K, const void *V, const void *Q_win, int dtype, const ecokv_shape *shape,
               const ecokv_params *params, const float *pre, float *scores, float *lambda, float *stats,
               void *workspace, size_t workspace_bytes, void *stream, bool noalloc)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_params(params))) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if (si.R > ECOKV_MAX_ROWS)
        return fail(ECOKV_EUNSUPPORTED, "(H_q/H_kv)*window = %d exceeds %d", si.R, ECOKV_MAX_ROWS);
    if (si.L == 0) return ECOKV_OK;
    if (!K || !Q_win || !scores) return fail(ECOKV_EINVAL, "K, Q_win and scores must be non-NULL");
    const bool vnorm = params->imp_mode == ECOKV_IMP_ATTN_VNORM;
    if (vnorm && !V) return fail(ECOKV_EINVAL, "imp_mode ECOKV_IMP_ATTN_VNORM needs V");
    const ecokv::WsLayout lay =
        ecokv::score_ws_layout(si.L, si.Hkv, si.B, si.D, si.R, si.Ptot, si.maxT, dtype == ECOKV_BF16, vnorm);
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < lay.total)
        return noalloc ? fail(ECOKV_EWORKSPACE,
                              "ecokv_score_noalloc: this call needs %zu bytes of scratch, the library holds %zu "
                              "per device; split it (fewer layers per call)", lay.total, workspace_bytes)
                       : fail(ECOKV_EWORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, lay.total);

    ecokv::ScoreArgs a;
    memset(&a, 0, sizeof a);
    a.K = K;
    a.V = vnorm ? V : nullptr;
    a.vnorm = vnorm ? 1 : 0;
    a.Q = Q_win;
    a.scores = scores;
    a.lambda = lambda;
    a.stats = stats;
    a.L = si.L;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.G = si.G;
    a.D = si.D;
    a.w = si.w;
    a.R = si.R;
    a.B = si.B;
    a.Ttot = si.Ttot;
    a.Ptot = si.Ptot;
    a.alpha = params->alpha;
    a.beta = params->beta;
    a.eps = params->eps;
    a.tau = params->tau > 0.f ? params->tau : sqrtf((float)si.D);
    a.inv_sqrt_d = 1.f / sqrtf((float)si.D);
    a.use_override = isnan(params->lambda_override) ? 0 : 1;
    a.lambda_override = a.use_override ? params->lambda_override : 0.f;
    a.pool_half = params->pool_kernel / 2;
    a.causal = params->causal;
    a.kbf16 = dtype == ECOKV_BF16;
    a.norm_mode = params->norm_mode;
    a.mad_tau = params->mad_tau;
    a.red_std = params->redundancy == ECOKV_RED_STD;
    a.centroid_prefix = params->centroid_scope == ECOKV_CENTROID_PREFIX;
    a.winsor_q = params->winsor_q;
    a.pre = pre;
    if (pre && ((uintptr_t)pre & 3u) != 0) return fail(ECOKV_EINVAL, "pre must be 4-byte aligned");
    // bounded waits between blocks poll up to this many times; ECOKV_SPIN_LIMIT
    // lowers it so that tests can make a wait give up (every kernel still ends)
    a.spin_limit = 1 << 20;
    if (const char *sl = getenv("ECOKV_SPIN_LIMIT")) a.spin_limit = atoi(sl);
    a.no_wait = noalloc ? 1 : 0;  // (its final step runs one block per unit: no waits, no status word)
    if ((rc = fill_seqtab(shape, nullptr, si.w, &a.seq, nullptr))) return rc;
    const hipError_t e = ecokv::score_launch(a, static_cast<char *>(workspace), lay, si.maxT,
                                             static_cast<hipStream_t>(stream), dtype == ECOKV_BF16);
    if (e != hipSuccess) return hip_fail(e, "ecokv_score launch");
    return ECOKV_OK;
}

}  // namespace

extern "C" {

int ecokv_prefill_workspace_size(const ecokv_shape *shape, size_t *bytes)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    if (si.R > ECOKV_MAX_ROWS)
        return fail(ECOKV_EUNSUPPORTED, "(H_q/H_kv)*window = %d exceeds %d", si.R, ECOKV_MAX_ROWS);
    // the element type changes the key block; report the larger
    const size_t b0 = ecokv::prefill_ws_bytes(si.L, si.Hkv, si.B, si.D, si.R, si.maxT, true);
    const size_t b1 = ecokv::prefill_ws_bytes(si.L, si.Hkv, si.B, si.D, si.R, si.maxT, false);
    *bytes = b0 > b1 ? b0 : b1;
    return ECOKV_OK;
}

int ecokv_prefill_write(const void *K_new, const void *V_new, const void *Q_win, int dtype, const ecokv_shape *shape,
                        const ecokv_params *params, void *K_cache, void *V_cache, float *pre, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_params(params))) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if (si.R > ECOKV_MAX_ROWS)
        return fail(ECOKV_EUNSUPPORTED, "(H_q/H_kv)*window = %d exceeds %d", si.R, ECOKV_MAX_ROWS);
    if (si.L == 0) return ECOKV_OK;
    if (!K_new || !Q_win || !K_cache || !pre) return fail(ECOKV_EINVAL, "K_new, Q_win, K_cache and pre must be non-NULL");
    if ((V_new == nullptr) != (V_cache == nullptr)) return fail(ECOKV_EINVAL, "V_new and V_cache: both or neither");
    const uintptr_t al = (uintptr_t)K_new | (uintptr_t)K_cache | (uintptr_t)V_new | (uintptr_t)V_cache;
    if ((al & 15u) != 0) return fail(ECOKV_EINVAL, "K_new, V_new, K_cache and V_cache must be 16-byte aligned");
    if (((uintptr_t)pre & 3u) != 0) return fail(ECOKV_EINVAL, "pre must be 4-byte aligned");
    // the copies read and write different memory
    const size_t es = dtype == ECOKV_BF16 ? 2 : 4;
    const size_t nb = (size_t)si.L * si.Hkv * (size_t)si.Ttot * si.D * es;
    auto overlap = [nb](const void *x, const void *y) {
        const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y;
        return a < b + nb && b < a + nb;
    };
    if (overlap(K_new, K_cache) || (V_new && (overlap(V_new, V_cache) || overlap(K_new, V_cache) ||
                                             overlap(V_new, K_cache) || overlap(K_cache, V_cache))))
        return fail(ECOKV_EINVAL, "the new rows and the cache must not overlap");
    const bool bf16 = dtype == ECOKV_BF16;
    const size_t need = ecokv::prefill_ws_bytes(si.L, si.Hkv, si.B, si.D, si.R, si.maxT, bf16);
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(ECOKV_EWORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);

    ecokv::ScoreArgs a;
    memset(&a, 0, sizeof a);
    a.K = K_cache;
    a.Ksrc = K_new;
    a.Q = Q_win;
    a.pre_out = pre;
    a.L = si.L;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.G = si.G;
    a.D = si.D;
    a.w = si.w;
    a.R = si.R;
    a.B = si.B;
    a.Ttot = si.Ttot;
    a.Ptot = si.Ptot;
    a.inv_sqrt_d = 1.f / sqrtf((float)si.D);
    a.causal = params->causal;
    a.kbf16 = bf16;
    if ((rc = fill_seqtab(shape, nullptr, si.w, &a.seq, nullptr))) return rc;
    const hipError_t e = ecokv::prefill_launch(a, V_new, V_cache, static_cast<char *>(workspace), si.maxT,
                                               static_cast<hipStream_t>(stream), bf16);
    if (e != hipSuccess) return hip_fail(e, "ecokv_prefill_write launch");
    return ECOKV_OK;
}

int ecokv_workspace_status(void *workspace, void *stream)
{
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned word = 0u;
    hipError_t e = hipMemcpyAsync(&word, workspace, sizeof word, hipMemcpyDeviceToHost, st);
    if (e == hipSuccess) e = hipStreamSynchronize(st);
    if (e != hipSuccess) return hip_fail(e, "ecokv_workspace_status");
    if (word == 0u) return ECOKV_OK;
    if ((e = ecokv::status_clear(static_cast<unsigned *>(workspace), st)) != hipSuccess)
        return hip_fail(e, "ecokv_workspace_status");
    return fail(ECOKV_ETIMEOUT,
                "a wait between the blocks of an ecokv_score call on this workspace gave up: that call's lambda "
                "and scores of the affected units are NaN");
}

int ecokv_index_count(const ecokv_shape *shape, const int32_t *budget, int64_t *count)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (!budget || !count) return fail(ECOKV_EINVAL, "budget and count must be non-NULL");
    ecokv::SeqTab t;
    int64_t per_lh = 0;
    if ((rc = fill_seqtab(shape, budget, si.w, &t, &per_lh))) return rc;
    *count = (int64_t)si.L * si.Hkv * per_lh;
    return ECOKV_OK;
}

int ecokv_index_count_mode(const ecokv_shape *shape, int mode, const int32_t *budget, int64_t *count)
{
    if (mode == ECOKV_PER_HEAD || mode == ECOKV_LAYER_FLAT) return ecokv_index_count(shape, budget, count);
    if (mode != ECOKV_HEAD_BUDGETS) return fail(ECOKV_EINVAL, "mode %d", mode);
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((!budget && (int64_t)si.L * si.Hkv > 0) || !count) return fail(ECOKV_EINVAL, "budget and count must be non-NULL");
    int64_t total = 0;
    if ((rc = head_budget_total(shape, si, budget, &total))) return rc;
    *count = total;
    return ECOKV_OK;
}

int ecokv_select_workspace_size(const ecokv_shape *shape, int mode, size_t *bytes)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_select_mode(si, mode))) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    int64_t groups = 0, maxn = 0;
    select_dims(si, shape, mode, &groups, &maxn);
    *bytes = ecokv::select_ws_layout(groups, maxn, mode != ECOKV_LAYER_FLAT).total;
    return ECOKV_OK;
}

int ecokv_select(const float *scores, const ecokv_shape *shape, int mode, const int32_t *budget,
                            int32_t *idx, int32_t *counts, int32_t *offsets, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_select_mode(si, mode))) return rc;
    if (!budget && (mode != ECOKV_HEAD_BUDGETS || (int64_t)si.L * si.Hkv > 0))
        return fail(ECOKV_EINVAL, "budget is NULL");
    ecokv::SelectArgs a;
    memset(&a, 0, sizeof a);
    int64_t per_lh = 0;
    if (mode == ECOKV_HEAD_BUDGETS) {
        int64_t total = 0;
        if ((rc = head_budget_total(shape, si, budget, &total))) return rc;
        if ((rc = fill_seqtab(shape, nullptr, si.w, &a.seq, &per_lh))) return rc;
        if (si.L == 0) return ECOKV_OK;
        if (!scores || !idx) return fail(ECOKV_EINVAL, "scores and idx must be non-NULL");
        if ((rc = select_workspace(si, shape, mode, workspace, workspace_bytes, &a))) return rc;
        a.scores = scores;
        a.idx = idx;
        a.counts = counts;
        a.offsets = offsets;
        a.L = si.L;
        a.Hkv = si.Hkv;
        a.B = si.B;
        a.w = si.w;
        a.Ptot = si.Ptot;
        a.heads = 1;
        // one launch per kLhChunk (layer, head) pairs, each with its table
        const int64_t npairs = (int64_t)si.L * si.Hkv;
        int64_t e0 = 0;
        for (int64_t lh0 = 0; lh0 < npairs; lh0 += ecokv::kLhChunk) {
            const int n = (int)(npairs - lh0 < ecokv::kLhChunk ? npairs - lh0 : ecokv::kLhChunk);
            e0 = fill_lhtab(shape, si.B, budget, lh0, n, e0, &a.lht);
            const hipError_t e = ecokv::select_launch(a, static_cast<char *>(workspace),
                                                      static_cast<hipStream_t>(stream));
            if (e != hipSuccess) return hip_fail(e, "ecokv_select launch");
        }
        return ECOKV_OK;
    }
    if ((rc = fill_seqtab(shape, budget, si.w, &a.seq, &per_lh))) return rc;
    if ((int64_t)si.L * si.Hkv * per_lh > INT32_MAX) return fail(ECOKV_EINVAL, "index count overflows int32");
    if (mode == ECOKV_LAYER_FLAT && (!counts || !offsets))
        return fail(ECOKV_EINVAL, "LAYER_FLAT needs counts and offsets");
    if (si.L == 0) return ECOKV_OK;
    if (!scores || !idx) return fail(ECOKV_EINVAL, "scores and idx must be non-NULL");
    if ((rc = select_workspace(si, shape, mode, workspace, workspace_bytes, &a))) return rc;
    a.scores = scores;
    a.idx = idx;
    a.counts = counts;
    a.offsets = offsets;
    a.L = si.L;
    a.Hkv = si.Hkv;
    a.B = si.B;
    a.w = si.w;
    a.Ptot = si.Ptot;
    a.per_lh = per_lh;
    a.flat = mode == ECOKV_LAYER_FLAT;
    const hipError_t e = ecokv::select_launch(a, static_cast<char *>(workspace), static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_select launch");
    return ECOKV_OK;
}

int ecokv_compact(const void *K, const void *V, int dtype, const ecokv_shape *shape, int mode, const int32_t *budget,
                  const int32_t *idx, const int32_t *counts, const int32_t *offsets, void *Kc, void *Vc,
                  void *stream)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if (mode != ECOKV_PER_HEAD && mode != ECOKV_LAYER_FLAT && mode != ECOKV_HEAD_BUDGETS)
        return fail(ECOKV_EINVAL, "mode %d", mode);
    if (!budget && (mode != ECOKV_HEAD_BUDGETS || (int64_t)si.L * si.Hkv > 0))
        return fail(ECOKV_EINVAL, "budget is NULL");
    ecokv::CompactArgs a;
    memset(&a, 0, sizeof a);
    int64_t per_lh = 0;
    if (mode == ECOKV_HEAD_BUDGETS) {
        int64_t total = 0;
        if ((rc = head_budget_total(shape, si, budget, &total))) return rc;
        if ((rc = fill_seqtab(shape, nullptr, si.w, &a.seq, &per_lh))) return rc;
        if (si.L == 0) return ECOKV_OK;
        if (!K || !V || !idx || !Kc || !Vc) return fail(ECOKV_EINVAL, "K, V, idx, Kc and Vc must be non-NULL");
        a.K = static_cast<const char *>(K);
        a.V = static_cast<const char *>(V);
        a.Kc = static_cast<char *>(Kc);
        a.Vc = static_cast<char *>(Vc);
        a.idx = idx;
        a.L = si.L;
        a.Hkv = si.Hkv;
        a.B = si.B;
        a.heads = 1;
        a.Ttot = si.Ttot;
        a.row_bytes = si.D * (dtype == ECOKV_BF16 ? 2 : 4);
        a.segs = a.row_bytes / 16;
        const int64_t npairs = (int64_t)si.L * si.Hkv;
        int64_t e0 = 0;
        for (int64_t lh0 = 0; lh0 < npairs; lh0 += ecokv::kLhChunk) {
            const int n = (int)(npairs - lh0 < ecokv::kLhChunk ? npairs - lh0 : ecokv::kLhChunk);
            a.e0 = e0;
            a.total = e0 = fill_lhtab(shape, si.B, budget, lh0, n, e0, &a.lht);
            const hipError_t e = ecokv::compact_launch(a, static_cast<hipStream_t>(stream));
            if (e != hipSuccess) return hip_fail(e, "ecokv_compact launch");
        }
        return ECOKV_OK;
    }
    if ((rc = fill_seqtab(shape, budget, si.w, &a.seq, &per_lh))) return rc;
    if (mode == ECOKV_LAYER_FLAT && !offsets) return fail(ECOKV_EINVAL, "LAYER_FLAT needs offsets");
    (void)counts;
    if (si.L == 0) return ECOKV_OK;
    if (!K || !V || !idx || !Kc || !Vc) return fail(ECOKV_EINVAL, "K, V, idx, Kc and Vc must be non-NULL");
    a.K = static_cast<const char *>(K);
    a.V = static_cast<const char *>(V);
    a.Kc = static_cast<char *>(Kc);
    a.Vc = static_cast<char *>(Vc);
    a.idx = idx;
    a.offsets = offsets;
    a.L = si.L;
    a.Hkv = si.Hkv;
    a.B = si.B;
    a.flat = mode == ECOKV_LAYER_FLAT;
    a.Ttot = si.Ttot;
    a.row_bytes = si.D * (dtype == ECOKV_BF16 ? 2 : 4);
    a.segs = a.row_bytes / 16;
    a.total = (int64_t)si.L * si.Hkv * per_lh;
    a.per_lh = per_lh;
    const hipError_t e = ecokv::compact_launch(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_compact launch");
    return ECOKV_OK;
}

int ecokv_decode_workspace_size(const ecokv_shape *shape, int32_t max_count, size_t *bytes)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    if (max_count < 1) return fail(ECOKV_EINVAL, "max_count %d < 1", max_count);
    *bytes = ecokv::decode_ws_bytes((int64_t)si.L * si.Hkv * si.B, si.G, si.D, max_count, false);
    return ECOKV_OK;
}

int ecokv_decode(const void *Q_dec, const void *Kc, const void *Vc, int dtype, const ecokv_shape *shape,
                 const int32_t *counts, const int32_t *offsets, int32_t max_count, float *O, float *lse,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if (max_count < 1) return fail(ECOKV_EINVAL, "max_count %d < 1", max_count);
    if (si.L == 0) return ECOKV_OK;
    // a smaller workspace than ecokv_decode_workspace_size says (one sized for
    // another max_count, say) will do down to `need`: fewer, longer chunks
    const size_t need = ecokv::decode_ws_bytes((int64_t)si.L * si.Hkv * si.B, si.G, si.D, max_count, true);
    if (!Q_dec || !Kc || !Vc || !counts || !offsets || !O)
        return fail(ECOKV_EINVAL, "Q_dec, Kc, Vc, counts, offsets and O must be non-NULL");
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (((uintptr_t)Q_dec & 15u) != 0 || ((uintptr_t)Kc & 15u) != 0 || ((uintptr_t)Vc & 15u) != 0)
        return fail(ECOKV_EINVAL, "Q_dec, Kc and Vc must be 16-byte aligned");
    if (workspace_bytes < need)
        return fail(ECOKV_EWORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
    ecokv::DecodeArgs a;
    memset(&a, 0, sizeof a);
    a.Q = Q_dec;
    a.Kc = Kc;
    a.Vc = Vc;
    a.counts = counts;
    a.offsets = offsets;
    a.O = O;
    a.lse = lse;
    a.L = si.L;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.G = si.G;
    a.B = si.B;
    a.D = si.D;
    a.max_count = max_count;
    a.qscale = 1.4426950408889634f / sqrtf((float)si.D);
    const hipError_t e = ecokv::decode_launch(a, static_cast<char *>(workspace), workspace_bytes, dtype == ECOKV_BF16,
                                             static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_decode launch");
    return ECOKV_OK;
}

int ecokv_rope_freqs(int rot_dim, double base, int kind, double stretch, double context, float *freq, float *factor)
{
    if (rot_dim < 2 || rot_dim % 2 != 0 || !freq || !factor)
        return fail(ECOKV_EINVAL, "rot_dim %d is not a positive even number, or freq or factor is NULL", rot_dim);
    if (kind < ECOKV_ROPE_PLAIN || kind > ECOKV_ROPE_BY_PARTS) return fail(ECOKV_EINVAL, "kind %d", kind);
    if (!(isfinite(base) && base > 1.0)) return fail(ECOKV_EINVAL, "base %g", base);
    if (kind != ECOKV_ROPE_PLAIN && !(isfinite(stretch) && stretch >= 1.0)) return fail(ECOKV_EINVAL, "stretch %g", stretch);
    if (kind == ECOKV_ROPE_BASE && rot_dim < 4) return fail(ECOKV_EINVAL, "rot_dim %d with a stretched base", rot_dim);
    if (kind == ECOKV_ROPE_BY_PARTS && !(isfinite(context) && context > 0.0)) return fail(ECOKV_EINVAL, "context %g", context);
    if (kind == ECOKV_ROPE_BASE) base *= pow(stretch, (double)rot_dim / (rot_dim - 2));
    if (!isfinite(base)) return fail(ECOKV_EINVAL, "the stretched base is not finite");
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (kind == ECOKV_ROPE_LINEAR) f /= stretch;
        if (kind == ECOKV_ROPE_BY_PARTS) {
            const double turns = context * f / 6.283185307179586477;
            const double keep = fmin(fmax((turns - 1.0) / 31.0, 0.0), 1.0);  // 1 turn .. 32 turns
            f *= keep + (1.0 - keep) / stretch;
        }
        freq[i] = (float)f;
    }
    *factor = kind == ECOKV_ROPE_BY_PARTS ? (float)(0.1 * log(stretch) + 1.0) : 1.f;
    return ECOKV_OK;
}

}  // extern "C"

namespace {

// Bytes [p, p + n) of an argument, and whether two share any.
struct Span {
    const void *p;
    size_t n;
};
bool overlap(const Span &x, const Span &y)
{
    const uintptr_t a = (uintptr_t)x.p, b = (uintptr_t)y.p;
    return x.p && y.p && x.n && y.n && a < b + y.n && b < a + x.n;
}

int check_rope(const ecokv_rope *r, int D)
{
    if (!r) return fail(ECOKV_EINVAL, "rope is NULL");
    if (r->rot_dim < 0 || r->rot_dim > D || r->rot_dim % 2 != 0)
        return fail(ECOKV_EINVAL, "rot_dim %d is not an even number in [0, %d]", r->rot_dim, D);
    if (r->rot_dim % 16 != 0) return fail(ECOKV_EUNSUPPORTED, "rot_dim %d (supported: multiples of 16)", r->rot_dim);
    if (r->interleaved != 0 && r->interleaved != 1) return fail(ECOKV_EINVAL, "interleaved must be 0 or 1");
    if (r->rot_dim > 0 && !r->freq) return fail(ECOKV_EINVAL, "freq is NULL");
    if (!isfinite(r->factor)) return fail(ECOKV_EINVAL, "factor %g", (double)r->factor);
    if (!(isfinite(r->norm_eps) && r->norm_eps >= 0.f)) return fail(ECOKV_EINVAL, "norm_eps %g", (double)r->norm_eps);
    if ((((uintptr_t)r->q_norm | (uintptr_t)r->k_norm) & 15u) != 0)
        return fail(ECOKV_EINVAL, "q_norm and k_norm must be 16-byte aligned");
    return ECOKV_OK;
}

// Rows of `tokens` tokens with `elems` elements of size es each, `stride`
// elements from token to token.
int check_rows(const void *p, int64_t stride, int64_t tokens, int64_t elems, int es, const char *name, Span *span)
{
    if (((uintptr_t)p & 15u) != 0) return fail(ECOKV_EINVAL, "%s must be 16-byte aligned", name);
    if (elems > INT32_MAX / 8) return fail(ECOKV_EINVAL, "a token of %s has %lld elements", name, (long long)elems);
    if (stride < elems || stride * es % 16 != 0 || stride > INT64_MAX / 4 / (tokens > 0 ? tokens : 1) / es)
        return fail(ECOKV_EINVAL, "the stride %lld of %s is below a token's %lld elements or no multiple of 16 bytes",
                    (long long)stride, name, (long long)elems);
    *span = Span{p, tokens > 0 ? (size_t)((tokens - 1) * stride + elems) * es : 0};
    return ECOKV_OK;
}

int check_tails(const ecokv_tails *t, const ShapeInfo &si, int es, ecokv::TailMap *m, Span *K, Span *V)
{
    if (!t) return fail(ECOKV_EINVAL, "tails is NULL");
    if (t->num_conts < 0 || t->num_pages < 1 || t->max_pages < 1)
        return fail(ECOKV_EINVAL, "tails: num_conts %d, num_pages %d, max_pages %d", t->num_conts, t->num_pages, t->max_pages);
    if (t->page_size < 1 || t->page_size > 65536 || (t->page_size & (t->page_size - 1)) != 0)
        return fail(ECOKV_EINVAL, "page_size %d is not a power of two of at most 65536", t->page_size);
    if ((int64_t)t->max_pages * t->page_size > INT32_MAX) return fail(ECOKV_EINVAL, "a tail of 2^31 rows or more");
    if (!t->K || !t->V || !t->table) return fail(ECOKV_EINVAL, "the tails' K, V and table must be non-NULL");
    if ((((uintptr_t)t->K | (uintptr_t)t->V) & 15u) != 0)
        return fail(ECOKV_EINVAL, "the tails' K and V must be 16-byte aligned");
    int shift = 0;
    while ((1 << shift) < t->page_size) ++shift;
    *m = ecokv::TailMap{t->table, t->num_conts, t->num_pages, shift, t->max_pages};
    const size_t n = (size_t)si.L * t->num_pages * si.Hkv * (size_t)t->page_size * si.D * es;
    *K = Span{t->K, n};
    *V = Span{t->V, n};
    return ECOKV_OK;
}

void fill_rope(const ecokv_rope *r, ecokv::RopeArgs *a)
{
    a->rot = r->rot_dim;
    a->interleaved = r->interleaved;
    a->freq = r->freq;
    a->factor = r->factor;
    a->eps = r->norm_eps;
    a->qw = r->q_norm;
    a->kw = r->k_norm;
}

int check_fan(const ShapeInfo &si, const int32_t *fan)
{
    if (!fan) return fail(ECOKV_EINVAL, "fan is NULL");
    if (fan[0] != 0) return fail(ECOKV_EINVAL, "fan[0] = %d, must be 0", fan[0]);
    for (int s = 0; s < si.B; ++s)
        if (fan[s + 1] < fan[s]) return fail(ECOKV_EINVAL, "fan[%d] = %d is below fan[%d] = %d", s + 1, fan[s + 1], s, fan[s]);
    if ((int64_t)(si.L > 0 ? si.L : 1) * si.Hq > (int64_t)INT32_MAX / (fan[si.B] > 0 ? fan[si.B] : 1))
        return fail(ECOKV_EINVAL, "too many (layer, query head, continuation) rows");
    return ECOKV_OK;
}

// Arguments of a call with num_nodes queries of each continuation; nodes: fan times
// num_nodes.
int check_tree(const ShapeInfo &si, const int32_t *fan, int32_t max_count, int32_t max_tail, int32_t num_nodes, int32_t *nodes)
{
    const int rc = check_fan(si, fan);
    if (rc) return rc;
    if (num_nodes < 1 || num_nodes > ECOKV_MAX_NODES)
        return fail(ECOKV_EINVAL, "num_nodes %d outside [1, %d]", num_nodes, ECOKV_MAX_NODES);
    if (max_count < 0 || max_tail < 0) return fail(ECOKV_EINVAL, "max_count %d or max_tail %d < 0", max_count, max_tail);
    if (max_tail > INT32_MAX - ECOKV_MAX_NODES) return fail(ECOKV_EINVAL, "max_tail %d", max_tail);
    if ((int64_t)(si.L > 0 ? si.L : 1) * si.Hq * num_nodes > (int64_t)INT32_MAX / (fan[si.B] > 0 ? fan[si.B] : 1))
        return fail(ECOKV_EINVAL, "too many (layer, query head, node) rows");
    for (int s = 0; s <= si.B; ++s) nodes[s] = fan[s] * num_nodes;
    return ECOKV_OK;
}

int check_tail_counts(const ecokv_tails *tails, int conts, const int32_t *tail_counts, int32_t max_tail)
{
    if (!tail_counts) return fail(ECOKV_EINVAL, "tail_counts must be non-NULL");
    if (tails->num_conts != conts) return fail(ECOKV_EINVAL, "the tails have %d continuations, the call %d", tails->num_conts, conts);
    if ((int64_t)max_tail > (int64_t)tails->max_pages * tails->page_size)
        return fail(ECOKV_EINVAL, "max_tail %d is more rows than %d pages of %d hold", max_tail, tails->max_pages,
                    tails->page_size);
    return ECOKV_OK;
}

// The masses of the tails' rows: one buffer, or two that do not overlap.
int check_tail_mass(const ecokv_tails *t, const ShapeInfo &si, const float *in, float *out)
{
    if (!in || !out) return fail(ECOKV_EINVAL, "tail_mass and tail_mass_out must be non-NULL");
    const size_t n = sizeof(float) * (size_t)si.L * t->num_pages * si.Hkv * (size_t)t->page_size;
    if (in != out && overlap(Span{in, n}, Span{out, n}))
        return fail(ECOKV_EINVAL, "tail_mass_out overlaps tail_mass and is not the same");
    return ECOKV_OK;
}

int check_evict(const ShapeInfo &si, int groups, int32_t max_rows, int32_t limit, int32_t keep, int32_t recent)
{
    if (max_rows < 0) return fail(ECOKV_EINVAL, "a bound of %d rows", max_rows);
    if (keep < 1 || limit < keep) return fail(ECOKV_EINVAL, "keep %d is below 1 or above the limit %d", keep, limit);
    if (recent < 0 || recent > keep) return fail(ECOKV_EINVAL, "recent %d outside [0, keep = %d]", recent, keep);
    if ((int64_t)si.L * si.Hkv * groups > INT32_MAX / 64) return fail(ECOKV_EINVAL, "too many (layer, KV head, group) units");
    return ECOKV_OK;
}

int evict_impl(ecokv::EvictArgs a, const ShapeInfo &si, int groups, int dtype, int32_t limit, int32_t keep, int32_t recent,
               const float *mass, float *mass_out, int32_t *new_counts, void *workspace, size_t workspace_bytes, void *stream)
{
    const int64_t words = ecokv::evict_plan_words(a.max_rows, keep);
    a.units = (int64_t)si.L * si.Hkv * groups;
    const size_t need = sizeof(int) * (size_t)a.units * (size_t)words;
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(ECOKV_EWORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
    a.mass = mass;
    a.mass_out = mass_out;
    a.new_counts = new_counts;
    a.plan = static_cast<int *>(workspace);
    a.Hkv = si.Hkv;
    a.groups = groups;
    a.row_bytes = si.D * (dtype == ECOKV_BF16 ? 2 : 4);
    a.limit = limit;
    a.keep = keep;
    a.recent = recent;
    a.cap = ecokv::evict_plan_cap(a.max_rows, keep);
    a.plan_stride = words;
    const hipError_t e = ecokv::evict_launch(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "eviction launch");
    return ECOKV_OK;
}

}  // namespace

extern "C" {

int ecokv_prefill_rope(const void *Q, int64_t q_stride, const void *K, int64_t k_stride, int dtype,
                       const ecokv_shape *shape, const ecokv_rope *rope, const int32_t *positions, void *Q_out,
                       void *K_out, void *Q_win, void *stream)
{
    ShapeInfo si;
    memset(&si, 0, sizeof si);
    int rc = check_heads(shape, &si);
    if (rc) return rc;
    if ((rc = check_seqs(shape, 0, &si))) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if ((rc = check_rope(rope, si.D))) return rc;
    if (Q_win)
        for (int s = 0; s < si.B; ++s)
            if (shape->window < 1 || shape->cu_seqlens[s + 1] - shape->cu_seqlens[s] < shape->window)
                return fail(ECOKV_EINVAL, "window %d is below 1 or longer than sequence %d", shape->window, s);
    if (si.L == 0) return ECOKV_OK;
    if ((K == nullptr) != (K_out == nullptr)) return fail(ECOKV_EINVAL, "K and K_out: both or neither");
    if ((Q == nullptr) != (Q_out == nullptr && Q_win == nullptr))
        return fail(ECOKV_EINVAL, "Q goes with Q_out, Q_win or both");
    const int es = dtype == ECOKV_BF16 ? 2 : 4;
    const int64_t tokens = (int64_t)si.L * si.Ttot, qe = (int64_t)si.Hq * si.D, ke = (int64_t)si.Hkv * si.D;
    Span q{}, k{};
    if (Q && (rc = check_rows(Q, q_stride, tokens, qe, es, "Q", &q))) return rc;
    if (K && (rc = check_rows(K, k_stride, tokens, ke, es, "K", &k))) return rc;
    const Span qo{Q_out, (size_t)(tokens * qe * es)}, ko{K_out, (size_t)(tokens * ke * es)},
        qw{Q_win, (size_t)(qe * si.L * si.B * (Q_win ? shape->window : 0) * es)};
    if ((((uintptr_t)Q_out | (uintptr_t)K_out | (uintptr_t)Q_win) & 15u) != 0)
        return fail(ECOKV_EINVAL, "Q_out, K_out and Q_win must be 16-byte aligned");
    // in place: a packed input onto itself
    const bool qi = Q && Q_out == Q && q_stride == qe, ki = K && K_out == K && k_stride == ke;
    if ((!qi && overlap(qo, q)) || (!ki && overlap(ko, k)) || overlap(qo, k) || overlap(ko, q) || overlap(qw, q) ||
        overlap(qw, k) || overlap(qo, ko) || overlap(qo, qw) || overlap(ko, qw))
        return fail(ECOKV_EINVAL, "an output overlaps an input or another output");
    if (!Q && !K) return ECOKV_OK;
    ecokv::RopeArgs a;
    memset(&a, 0, sizeof a);
    a.Q = static_cast<const char *>(Q);
    a.K = static_cast<const char *>(K);
    a.Qo = static_cast<char *>(Q_out);
    a.Ko = static_cast<char *>(K_out);
    a.win = static_cast<char *>(Q_win);
    a.q_stride = q_stride * es;
    a.k_stride = k_stride * es;
    a.positions = positions;
    fill_rope(rope, &a);
    a.L = si.L;
    a.n = (int)si.Ttot;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.B = si.B;
    a.w = shape->window;
    a.hq = Q ? si.Hq : 0;
    a.hk = K ? si.Hkv : 0;
    if ((rc = fill_seqtab(shape, nullptr, 0, &a.seq, nullptr))) return rc;
    const hipError_t e = ecokv::rope_launch(a, false, dtype == ECOKV_BF16, si.D, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_prefill_rope launch");
    return ECOKV_OK;
}

int ecokv_append(const void *Q_new, int64_t q_stride, const void *K_new, int64_t k_stride, const void *V_new,
                 int64_t v_stride, int dtype, const ecokv_shape *shape, const ecokv_rope *rope,
                 const int32_t *positions, const int32_t *conts, const int32_t *rows, int32_t num_tokens,
                 const ecokv_tails *tails, void *Q_dec, void *stream)
{
    ShapeInfo si;
    memset(&si, 0, sizeof si);
    int rc = check_heads(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if ((rc = check_rope(rope, si.D))) return rc;
    if (num_tokens < 0) return fail(ECOKV_EINVAL, "num_tokens %d < 0", num_tokens);
    if (si.L == 0 || num_tokens == 0) return ECOKV_OK;
    const int es = dtype == ECOKV_BF16 ? 2 : 4;
    ecokv::RopeArgs a;
    memset(&a, 0, sizeof a);
    Span tk{}, tv{}, q{}, k{}, v{};
    if ((rc = check_tails(tails, si, es, &a.map, &tk, &tv))) return rc;
    if (!K_new || !V_new || !positions || !rows)
        return fail(ECOKV_EINVAL, "K_new, V_new, positions and rows must be non-NULL");
    if ((Q_new == nullptr) != (Q_dec == nullptr)) return fail(ECOKV_EINVAL, "Q_new and Q_dec: both or neither");
    if (!conts && num_tokens > tails->num_conts)
        return fail(ECOKV_EINVAL, "without conts, %d tokens need as many continuations (%d)", num_tokens, tails->num_conts);
    const int64_t tokens = (int64_t)si.L * num_tokens, qe = (int64_t)si.Hq * si.D, ke = (int64_t)si.Hkv * si.D;
    if (Q_new && (rc = check_rows(Q_new, q_stride, tokens, qe, es, "Q_new", &q))) return rc;
    if ((rc = check_rows(K_new, k_stride, tokens, ke, es, "K_new", &k))) return rc;
    if ((rc = check_rows(V_new, v_stride, tokens, ke, es, "V_new", &v))) return rc;
    if (((uintptr_t)Q_dec & 15u) != 0) return fail(ECOKV_EINVAL, "Q_dec must be 16-byte aligned");
    const Span out[3] = {tk, tv, Span{Q_dec, (size_t)(tokens * qe * es)}}, in[3] = {q, k, v};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j)
            if (overlap(out[i], in[j]) || (i < j && overlap(out[i], out[j])))
                return fail(ECOKV_EINVAL, "the tails, Q_dec and the new rows must not overlap");
    a.Q = static_cast<const char *>(Q_new);
    a.K = static_cast<const char *>(K_new);
    a.V = static_cast<const char *>(V_new);
    a.Qo = static_cast<char *>(Q_dec);
    a.Ko = static_cast<char *>(tails->K);
    a.Vo = static_cast<char *>(tails->V);
    a.q_stride = q_stride * es;
    a.k_stride = k_stride * es;
    a.v_stride = v_stride * es;
    a.positions = positions;
    a.conts = conts;
    a.rows = rows;
    fill_rope(rope, &a);
    a.L = si.L;
    a.n = num_tokens;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.B = 1;
    a.hq = Q_new ? si.Hq : 0;
    a.hk = si.Hkv;
    const hipError_t e = ecokv::rope_launch(a, true, dtype == ECOKV_BF16, si.D, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_append launch");
    return ECOKV_OK;
}

int ecokv_decode_shared_workspace_size(const ecokv_shape *shape, const int32_t *fan, int32_t max_count,
                                       int32_t max_tail, size_t *bytes)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_fan(si, fan))) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    if (max_count < 0 || max_tail < 0) return fail(ECOKV_EINVAL, "max_count %d or max_tail %d < 0", max_count, max_tail);
    // the element type changes the split; report the larger
    const size_t b0 = ecokv::shared_grid((int64_t)si.L * si.Hkv, si.G, si.D, si.B, fan, max_count, max_tail, true).bytes;
    const size_t b1 = ecokv::shared_grid((int64_t)si.L * si.Hkv, si.G, si.D, si.B, fan, max_count, max_tail, false).bytes;
    *bytes = b0 > b1 ? b0 : b1;
    return ECOKV_OK;
}

int ecokv_decode_shared(const void *Q_dec, const void *Kc, const void *Vc, int dtype, const ecokv_shape *shape,
                        const int32_t *fan, const int32_t *counts, const int32_t *offsets, int32_t max_count,
                        const ecokv_tails *tails, const int32_t *tail_counts, int32_t max_tail, float *O, float *lse,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if ((rc = check_fan(si, fan))) return rc;
    if (max_count < 0 || max_tail < 0) return fail(ECOKV_EINVAL, "max_count %d or max_tail %d < 0", max_count, max_tail);
    if (si.L == 0 || fan[si.B] == 0) return ECOKV_OK;
    ecokv::SharedArgs a;
    memset(&a, 0, sizeof a);
    if (!Q_dec || !O) return fail(ECOKV_EINVAL, "Q_dec and O must be non-NULL");
    if (max_count > 0 && (!Kc || !Vc || !counts || !offsets))
        return fail(ECOKV_EINVAL, "Kc, Vc, counts and offsets must be non-NULL");
    if ((((uintptr_t)Q_dec | (uintptr_t)Kc | (uintptr_t)Vc | (uintptr_t)O) & 15u) != 0)
        return fail(ECOKV_EINVAL, "Q_dec, Kc, Vc and O must be 16-byte aligned");
    if (max_tail > 0) {
        Span tk, tv;
        if ((rc = check_tails(tails, si, dtype == ECOKV_BF16 ? 2 : 4, &a.map, &tk, &tv))) return rc;
        if (!tail_counts) return fail(ECOKV_EINVAL, "tail_counts must be non-NULL");
        if (tails->num_conts != fan[si.B])
            return fail(ECOKV_EINVAL, "the tails have %d continuations, fan %d", tails->num_conts, fan[si.B]);
        if ((int64_t)max_tail > (int64_t)tails->max_pages * tails->page_size)
            return fail(ECOKV_EINVAL, "max_tail %d is more rows than %d pages of %d hold", max_tail, tails->max_pages,
                        tails->page_size);
    }
    a.grid = ecokv::shared_grid((int64_t)si.L * si.Hkv, si.G, si.D, si.B, fan, max_count, max_tail,
                                dtype == ECOKV_BF16);
    if (a.grid.prompt_blocks > INT32_MAX - (1 << 20) || a.grid.tail_waves > INT32_MAX - (1 << 20))
        return fail(ECOKV_EINVAL, "too many parts of kept rows or tails");
    if (!workspace && a.grid.bytes > 0) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < a.grid.bytes)
        return fail(ECOKV_EWORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, a.grid.bytes);
    a.Q = static_cast<const char *>(Q_dec);
    a.Kc = static_cast<const char *>(Kc);
    a.Vc = static_cast<const char *>(Vc);
    a.Kt = max_tail > 0 ? static_cast<const char *>(tails->K) : nullptr;
    a.Vt = max_tail > 0 ? static_cast<const char *>(tails->V) : nullptr;
    a.counts = counts;
    a.offsets = offsets;
    a.tail_counts = tail_counts;
    a.O = O;
    a.lse = lse;
    // (the sums first: they stay 16-byte aligned)
    a.acc = static_cast<float *>(workspace);
    a.ms = reinterpret_cast<float2 *>(a.acc + (size_t)(a.grid.np + a.grid.nt) * (size_t)a.grid.qrows * si.D);
    a.L = si.L;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.G = si.G;
    a.B = si.B;
    a.N = fan[si.B];
    a.D = si.D;
    a.max_count = max_count;
    a.max_tail = max_tail;
    a.qscale = 1.4426950408889634f / sqrtf((float)si.D);
    for (int s = 0; s <= si.B; ++s) a.fan[s] = fan[s];
    const hipError_t e = ecokv::shared_launch(a, dtype == ECOKV_BF16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_decode_shared launch");
    return ECOKV_OK;
}

int ecokv_tree_masks(int num_nodes, const int32_t *parents, uint64_t *masks, int32_t *depths)
{
    if (num_nodes < 1 || num_nodes > ECOKV_MAX_NODES)
        return fail(ECOKV_EINVAL, "num_nodes %d outside [1, %d]", num_nodes, ECOKV_MAX_NODES);
    if (!parents || !masks) return fail(ECOKV_EINVAL, "parents and masks must be non-NULL");
    for (int i = 0; i < num_nodes; ++i)
        if (parents[i] < -1 || parents[i] >= i)
            return fail(ECOKV_EINVAL, "parents[%d] = %d is neither -1 nor an earlier node", i, parents[i]);
    for (int i = 0; i < num_nodes; ++i) {
        const int p = parents[i];
        masks[i] = (p >= 0 ? masks[p] : 0) | (uint64_t)1 << i;
        if (depths) depths[i] = p >= 0 ? depths[p] + 1 : 0;
    }
    return ECOKV_OK;
}

int ecokv_decode_tree_workspace_size(const ecokv_shape *shape, const int32_t *fan, int32_t max_count, int32_t max_tail,
                                     int32_t num_nodes, size_t *bytes)
{
    ShapeInfo si;
    int32_t nodes[ECOKV_MAX_SEQS + 1];
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if ((rc = check_tree(si, fan, max_count, max_tail, num_nodes, nodes))) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    ecokv::TreeTails tails;
    ecokv::TreeEven even;
    *bytes = 0;
    for (int bf16 = 0; bf16 < 2; ++bf16) {  // the element type changes the split; report the larger
        const size_t n = ecokv::tree_grid((int64_t)si.L * si.Hkv, si.G, si.D, si.B, nodes, fan[si.B], num_nodes, max_count,
                                          max_tail, bf16 != 0, &tails, &even).bytes;
        if (n > *bytes) *bytes = n;
    }
    return ECOKV_OK;
}

int ecokv_decode_tree(const void *Q_dec, const void *Kc, const void *Vc, int dtype, const ecokv_shape *shape,
                      const int32_t *fan, const int32_t *counts, const int32_t *offsets, int32_t max_count,
                      const ecokv_tails *tails, const int32_t *tail_counts, int32_t max_tail, int32_t num_nodes,
                      const uint64_t *masks, void *O, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    ecokv::TreeArgs a;
    memset(&a, 0, sizeof a);
    ecokv::SharedArgs &s = a.s;
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if ((rc = check_tree(si, fan, max_count, max_tail, num_nodes, s.fan))) return rc;
    if (si.L == 0 || fan[si.B] == 0) return ECOKV_OK;
    const bool bf16 = dtype == ECOKV_BF16;
    const size_t rows = (size_t)si.L * si.Hq * s.fan[si.B], q = rows * si.D * (bf16 ? 2 : 4);
    if (!Q_dec || !O || !masks) return fail(ECOKV_EINVAL, "Q_dec, masks and O must be non-NULL");
    if (max_count > 0 && (!Kc || !Vc || !counts || !offsets))
        return fail(ECOKV_EINVAL, "Kc, Vc, counts and offsets must be non-NULL");
    if ((((uintptr_t)Q_dec | (uintptr_t)Kc | (uintptr_t)Vc | (uintptr_t)O) & 15u) != 0)
        return fail(ECOKV_EINVAL, "Q_dec, Kc, Vc and O must be 16-byte aligned");
    Span tk, tv;
    if ((rc = check_tails(tails, si, bf16 ? 2 : 4, &s.map, &tk, &tv))) return rc;
    if ((rc = check_tail_counts(tails, fan[si.B], tail_counts, max_tail))) return rc;
    const Span so{O, q}, sl{lse, rows * 4}, sw{workspace, workspace_bytes}, in[3] = {Span{Q_dec, q}, tk, tv};
    for (int i = 0; i < 3; ++i)
        if (overlap(in[i], so) || overlap(in[i], sl) || overlap(in[i], sw))
            return fail(ECOKV_EINVAL, "O, lse or the workspace overlaps Q_dec or the tails");
    if (overlap(so, sl) || overlap(so, sw) || overlap(sl, sw)) return fail(ECOKV_EINVAL, "O, lse and the workspace overlap");
    s.grid = ecokv::tree_grid((int64_t)si.L * si.Hkv, si.G, si.D, si.B, s.fan, fan[si.B], num_nodes, max_count, max_tail, bf16,
                              &a.tails, &a.even);
    if (s.grid.prompt_blocks > INT32_MAX - (1 << 20) || s.grid.tail_waves > INT32_MAX - (1 << 20) ||
        a.tails.blocks > INT32_MAX - (1 << 20) - s.grid.prompt_blocks)
        return fail(ECOKV_EINVAL, "too many parts of kept rows or tails");
    if (!workspace) return fail(ECOKV_EINVAL, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(ECOKV_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < s.grid.bytes)
        return fail(ECOKV_EWORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, s.grid.bytes);
    s.Q = static_cast<const char *>(Q_dec);
    s.Kc = static_cast<const char *>(Kc);
    s.Vc = static_cast<const char *>(Vc);
    s.Kt = static_cast<const char *>(tails->K);
    s.Vt = static_cast<const char *>(tails->V);
    s.counts = counts;
    s.offsets = offsets;
    s.tail_counts = tail_counts;
    s.O = static_cast<float *>(O);
    s.lse = lse;
    s.acc = static_cast<float *>(workspace);
    s.ms = reinterpret_cast<float2 *>(s.acc + (size_t)(s.grid.np + s.grid.nt) * (size_t)s.grid.qrows * si.D);
    s.part_steps = a.even.fill ? reinterpret_cast<int *>(s.ms + (size_t)(s.grid.np + s.grid.nt) * (size_t)s.grid.qrows) : nullptr;
    s.L = si.L;
    s.Hq = si.Hq;
    s.Hkv = si.Hkv;
    s.G = si.G;
    s.B = si.B;
    s.N = s.fan[si.B];
    s.D = si.D;
    s.max_count = max_count;
    s.max_tail = max_tail;
    s.qscale = 1.4426950408889634f / sqrtf((float)si.D);
    s.nodes = num_nodes;
    s.bf16 = bf16;
    s.tree_rows = a.tails.rows;
    a.masks = reinterpret_cast<const unsigned long long *>(masks);
    a.conts = fan[si.B];
    const hipError_t e = ecokv::tree_launch(a, bf16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_decode_tree launch");
    return ECOKV_OK;
}

}  // extern "C"

namespace {

int commit_impl(int dtype, const ecokv_shape *shape, const ecokv_tails *tails, const int32_t *tail_counts, int32_t num_nodes,
                const int32_t *path, const int32_t *accepted, int32_t *taken, bool tells, void *stream)
{
    ShapeInfo si;
    memset(&si, 0, sizeof si);
    int rc = check_heads(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if (num_nodes < 1 || num_nodes > ECOKV_MAX_NODES)
        return fail(ECOKV_EINVAL, "num_nodes %d outside [1, %d]", num_nodes, ECOKV_MAX_NODES);
    ecokv::CommitArgs a;
    memset(&a, 0, sizeof a);
    Span tk, tv;
    if (si.L == 0) return ECOKV_OK;
    const int es = dtype == ECOKV_BF16 ? 2 : 4;
    if ((rc = check_tails(tails, si, es, &a.map, &tk, &tv))) return rc;
    if (overlap(tk, tv)) return fail(ECOKV_EINVAL, "the tails' K and V overlap");
    if (!tail_counts || !path || !accepted) return fail(ECOKV_EINVAL, "tail_counts, path and accepted must be non-NULL");
    if (tells && !taken) return fail(ECOKV_EINVAL, "taken must be non-NULL");
    const size_t n = 4 * (size_t)tails->num_conts;
    const Span in[5] = {tk, tv, Span{tail_counts, n}, Span{path, n * num_nodes}, Span{accepted, n}};
    for (int i = 0; tells && i < 5; ++i)
        if (overlap(in[i], Span{taken, n})) return fail(ECOKV_EINVAL, "taken overlaps what the call reads or the tails");
    a.units = (int64_t)si.L * si.Hkv * tails->num_conts;
    if (a.units == 0) return ECOKV_OK;
    if (a.units > INT32_MAX / 4) return fail(ECOKV_EINVAL, "too many (layer, KV head, continuation) units");
    a.K = static_cast<char *>(tails->K);
    a.V = static_cast<char *>(tails->V);
    a.tail_counts = tail_counts;
    a.path = path;
    a.accepted = accepted;
    a.taken = tells ? taken : nullptr;
    a.Hkv = si.Hkv;
    a.N = tails->num_conts;
    a.nodes = num_nodes;
    a.row_bytes = si.D * es;
    const hipError_t e = ecokv::commit_launch(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_commit launch");
    return ECOKV_OK;
}

}  // namespace

extern "C" {

int ecokv_commit(int dtype, const ecokv_shape *shape, const ecokv_tails *tails, const int32_t *tail_counts,
                 int32_t num_nodes, const int32_t *path, const int32_t *accepted, void *stream)
{
    return commit_impl(dtype, shape, tails, tail_counts, num_nodes, path, accepted, nullptr, false, stream);
}

int ecokv_commit_taken(int dtype, const ecokv_shape *shape, const ecokv_tails *tails, const int32_t *tail_counts,
                       int32_t num_nodes, const int32_t *path, const int32_t *accepted, int32_t *taken, void *stream)
{
    return commit_impl(dtype, shape, tails, tail_counts, num_nodes, path, accepted, taken, true, stream);
}

int ecokv_accumulate(const void *Q_dec, const float *lse, const void *Kc, int dtype, const ecokv_shape *shape,
                     const int32_t *fan, const int32_t *counts, const int32_t *offsets, int32_t max_count,
                     const ecokv_tails *tails, const int32_t *tail_counts, int32_t max_tail, int32_t num_nodes,
                     const int32_t *path, const int32_t *accepted, float decay, const float *mass, const float *tail_mass,
                     float *mass_out, float *tail_mass_out, void *stream)
{
    ShapeInfo si;
    ecokv::MassArgs a;
    memset(&a, 0, sizeof a);
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    int32_t nodes[ECOKV_MAX_SEQS + 1];
    if ((rc = check_tree(si, fan, max_count, max_tail, num_nodes, nodes))) return rc;
    if (!(isfinite(decay) && decay >= 0.f)) return fail(ECOKV_EINVAL, "decay %g", (double)decay);
    if ((path == nullptr) != (accepted == nullptr)) return fail(ECOKV_EINVAL, "path and accepted: both or neither");
    if (!path && num_nodes != 1) return fail(ECOKV_EINVAL, "%d queries of a continuation need path and accepted", num_nodes);
    const int N = fan[si.B];
    if (si.L == 0 || (max_count == 0 && (max_tail == 0 || N == 0))) return ECOKV_OK;
    if (N > 0 && (!Q_dec || !lse)) return fail(ECOKV_EINVAL, "Q_dec and lse must be non-NULL");
    if (max_count > 0 && (!Kc || !counts || !offsets || !mass || !mass_out))
        return fail(ECOKV_EINVAL, "Kc, counts, offsets, mass and mass_out must be non-NULL");
    if ((((uintptr_t)Q_dec | (uintptr_t)Kc) & 15u) != 0) return fail(ECOKV_EINVAL, "Q_dec and Kc must be 16-byte aligned");
    const bool bf16 = dtype == ECOKV_BF16;
    const bool tailed = max_tail > 0 && N > 0;
    if (tailed) {
        Span tk, tv;
        if ((rc = check_tails(tails, si, bf16 ? 2 : 4, &a.map, &tk, &tv))) return rc;
        if ((rc = check_tail_counts(tails, N, tail_counts, max_tail))) return rc;
        if ((rc = check_tail_mass(tails, si, tail_mass, tail_mass_out))) return rc;
    }
    a.Q = static_cast<const char *>(Q_dec);
    a.lse = lse;
    a.Kc = static_cast<const char *>(Kc);
    a.Kt = tailed ? static_cast<const char *>(tails->K) : nullptr;
    a.counts = counts;
    a.offsets = offsets;
    a.tail_counts = tail_counts;
    a.path = path;
    a.accepted = accepted;
    a.mass = mass;
    a.tail_mass = tail_mass;
    a.mass_out = mass_out;
    a.tail_mass_out = tail_mass_out;
    a.L = si.L;
    a.Hq = si.Hq;
    a.Hkv = si.Hkv;
    a.G = si.G;
    a.B = si.B;
    a.N = N;
    a.D = si.D;
    a.nodes = num_nodes;
    a.max_count = max_count;
    a.max_tail = max_tail;
    a.decay = decay;
    const double scale = 1.4426950408889634074 / sqrt((double)si.D);
    a.scale = (float)scale;
    a.scale_rest = (float)(scale / a.scale - 1.0);
    for (int s = 0; s <= si.B; ++s) a.fan[s] = fan[s];
    ecokv::mass_grid((int64_t)si.L * si.Hkv, si.B, tailed ? N : 0, max_count, max_tail, &a.kept_parts, &a.tail_parts,
                     &a.kept_blocks, &a.tail_blocks);
    if (a.kept_blocks > INT32_MAX - (1 << 20) || a.tail_blocks > INT32_MAX - (1 << 20) - a.kept_blocks)
        return fail(ECOKV_EINVAL, "too many parts of kept rows or tails");
    const hipError_t e = ecokv::mass_launch(a, bf16, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "ecokv_accumulate launch");
    return ECOKV_OK;
}

int ecokv_evict_workspace_size(const ecokv_shape *shape, int32_t groups, int32_t max_rows, int32_t keep, size_t *bytes)
{
    ShapeInfo si;
    memset(&si, 0, sizeof si);
    const int rc = check_heads(shape, &si);
    if (rc) return rc;
    if (!bytes) return fail(ECOKV_EINVAL, "bytes is NULL");
    if (groups < 0) return fail(ECOKV_EINVAL, "groups %d < 0", groups);
    if (max_rows < 0 || keep < 1) return fail(ECOKV_EINVAL, "max_rows %d < 0 or keep %d < 1", max_rows, keep);
    *bytes = sizeof(int) * (size_t)si.L * si.Hkv * groups * (size_t)ecokv::evict_plan_words(max_rows, keep);
    return ECOKV_OK;
}

int ecokv_evict(void *Kc, void *Vc, int dtype, const ecokv_shape *shape, const int32_t *counts, const int32_t *offsets,
                int32_t max_count, int32_t limit, int32_t keep, int32_t recent, const float *mass, float *mass_out,
                int32_t *new_counts, void *workspace, size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    ecokv::EvictArgs a;
    memset(&a, 0, sizeof a);
    int rc = check_shape(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if ((rc = check_evict(si, si.B, max_count, limit, keep, recent))) return rc;
    if (si.L == 0) return ECOKV_OK;
    if (!Kc || !Vc || !counts || !offsets || !mass || !mass_out || !new_counts)
        return fail(ECOKV_EINVAL, "Kc, Vc, counts, offsets, mass, mass_out and new_counts must be non-NULL");
    if ((((uintptr_t)Kc | (uintptr_t)Vc) & 15u) != 0) return fail(ECOKV_EINVAL, "Kc and Vc must be 16-byte aligned");
    a.K = static_cast<char *>(Kc);
    a.V = static_cast<char *>(Vc);
    a.counts = counts;
    a.offsets = offsets;
    a.max_rows = max_count;
    return evict_impl(a, si, si.B, dtype, limit, keep, recent, mass, mass_out, new_counts, workspace, workspace_bytes, stream);
}

int ecokv_evict_tails(int dtype, const ecokv_shape *shape, const ecokv_tails *tails, const int32_t *tail_counts,
                      int32_t max_tail, int32_t limit, int32_t keep, int32_t recent, const float *tail_mass,
                      float *tail_mass_out, int32_t *new_counts, void *workspace, size_t workspace_bytes, void *stream)
{
    ShapeInfo si;
    memset(&si, 0, sizeof si);
    ecokv::EvictArgs a;
    memset(&a, 0, sizeof a);
    int rc = check_heads(shape, &si);
    if (rc) return rc;
    if (dtype != ECOKV_BF16 && dtype != ECOKV_F32) return fail(ECOKV_EUNSUPPORTED, "dtype %d", dtype);
    if (si.L == 0) return ECOKV_OK;
    Span tk, tv;
    if ((rc = check_tails(tails, si, dtype == ECOKV_BF16 ? 2 : 4, &a.map, &tk, &tv))) return rc;
    if (overlap(tk, tv)) return fail(ECOKV_EINVAL, "the tails' K and V overlap");
    if ((rc = check_evict(si, tails->num_conts, max_tail, limit, keep, recent))) return rc;
    if ((rc = check_tail_counts(tails, tails->num_conts, tail_counts, max_tail))) return rc;
    if ((rc = check_tail_mass(tails, si, tail_mass, tail_mass_out))) return rc;
    if (!new_counts) return fail(ECOKV_EINVAL, "new_counts must be non-NULL");
    if (tails->num_conts == 0) return ECOKV_OK;
    a.K = static_cast<char *>(tails->K);
    a.V = static_cast<char *>(tails->V);
    a.counts = tail_counts;
    a.tails = 1;
    a.max_rows = max_tail;
    return evict_impl(a, si, tails->num_conts, dtype, limit, keep, recent, tail_mass, tail_mass_out, new_counts, workspace,
                      workspace_bytes, stream);
}

int ecokv_pyramid_budgets(int num_layers, double total, double beta, int window, int32_t *out)
{
    if (num_layers < 1 || !out) return fail(ECOKV_EINVAL, "num_layers %d < 1 or out is NULL", num_layers);
    if (!(isfinite(total) && total > 0.0) || !(isfinite(beta) && beta > 0.0))
        return fail(ECOKV_EINVAL, "total %g and beta %g must be positive and finite", total, beta);
    if (window < 1) return fail(ECOKV_EINVAL, "window %d < 1", window);
    const int m = num_layers;
    const double last = total / (beta * m), first = 2.0 * total / m - last;
    // every value checked before any is written
    for (int pass = 0; pass < 2; ++pass)
        for (int l = 0; l < m; ++l) {
            const double v = m == 1 ? total : first - (first - last) * l / (m - 1);
            // rounded down; a value within 1e-9 below an integer is that integer
            const double f = floor(v + 1e-9);
            if (pass == 0 && !(f >= window && f <= (double)INT32_MAX))
                return fail(ECOKV_EINVAL, "layer %d budget %g is outside [window %d, INT32_MAX]", l, v, window);
            if (pass == 1) out[l] = (int32_t)f;
        }
    return ECOKV_OK;
}

const char *ecokv_last_error(void) { return g_err; }

}  // extern "C"
