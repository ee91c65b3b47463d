"""ecokv_prefill_rope and ecokv_append against the formulas in 64 bits, for
both pair layouts, every part of the head, with and without norms, packed and
strided inputs, far positions; what a call must leave alone.

Tolerance.  In float32 a normed element is off by at most 16 roundings (a sum of
D squares over 8 serial and 5 tree steps, the root, two products), 16 * 2^-24;
a cosine or sine by the rounding of its reduced angle (2^-25 half turns, 2^-23.3
radians), two steps of the function and one of the factor: 2^-22.  So
  |y - y64| <= u |y64| + 2^-19 (|a| + |b|) factor,
u half a step of the element type (bf16 2^-8, fp32 2^-24), a and b the normed
pair; 2^-19 |y64| instead of the second term outside the rotated part.
"""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-rope] {msg}", file=sys.stderr, flush=True)


def turned(x, positions, freq, rot, inter, factor, weight, eps):
    """x [..., n, H, D] in 64 bits, and the tolerance's second term beside the result."""
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    y, slack = x.clone(), x.abs()
    if rot:
        th = positions.double()[:, None] * freq.double()
        c, s = (factor * th.cos())[:, None, :], (factor * th.sin())[:, None, :]
        ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        slack[..., ia] = slack[..., ib] = (a.abs() + b.abs()) * abs(factor)
    return y, slack


def near(got, want, slack, dtype):
    bound = HALF_STEP[dtype] * want.abs() + 2.0 ** -19 * slack
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), f"worst {float((err / bound.clamp_min(1e-300)).max()):.3f} of the tolerance"


def make(seed, dtype, L, n, Hq, Hkv, D, rot, norm, fused=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    if fused:
        x = r(L, n, Hq + 2 * Hkv, D).to(TYPES[dtype])
        Q, K, V = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    else:
        Q, K, V = (r(L, n, h, D).to(TYPES[dtype]) for h in (Hq, Hkv, Hkv))
    freq = (10000.0 ** (-2 * torch.arange(rot // 2, dtype=torch.float64) / max(rot, 1))).float().cuda()
    w = [(1 + 0.2 * r(D)).to(TYPES[dtype]) if norm else None for _ in range(2)]
    return Q, K, V, freq, w


CASES = [  # dtype, D, Hq, Hkv, rot, interleaved, norm, factor, L, sequences, window
    ("bf16", 128, 28, 4, 128, False, False, 1.0, 1, [700], 4),
    ("bf16", 128, 32, 8, 128, True, True, 1.14, 2, [33, 1, 257], 1),
    ("bf16", 128, 7, 1, 96, False, True, 1.0, 1, [5, 130], 5),
    ("bf16", 64, 12, 12, 64, False, False, 1.0, 3, [61, 64], 8),
    ("bf16", 64, 2, 2, 16, True, False, -0.5, 1, [1], 1),
    ("f32", 128, 8, 4, 128, False, True, 1.0, 1, [301], 8),
    ("f32", 128, 3, 1, 48, True, False, 1.0, 2, [17, 16], 16),
    ("f32", 64, 16, 2, 32, False, True, 1.3, 1, [1, 2, 3, 513], 1),
    ("f32", 64, 5, 5, 0, False, True, 1.0, 1, [90], 2),
    ("bf16", 128, 4, 2, 0, True, False, 1.0, 1, [90], 2),
]


@pytest.mark.parametrize("far", [None, 0, 1_000_003, 2 ** 31 - 1000])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:7])))
def test_prefill_rope(case, far):
    import paper_2609_06663_amd as P
    dtype, D, Hq, Hkv, rot, inter, norm, factor, L, lens, w = case
    say(f"{case} positions from {far}")
    cu = [0] + list(np.cumsum(lens))
    n = cu[-1]
    Q, K, _, freq, wt = make(11, dtype, L, n, Hq, Hkv, D, rot, norm)
    own = torch.cat([torch.arange(t) for t in lens]).int().cuda()
    pos = own if far is None else own + far
    rope = P.Rope(rot, freq, inter, factor, *wt, 1e-5)
    shape = P.Shape(L, Hq, Hkv, D, w, cu)
    out = lambda *s: torch.full(s, 7.0, dtype=TYPES[dtype], device="cuda")
    Qo, Ko, Qw = out(L, n, Hq, D), out(L, n, Hkv, D), out(L, Hq, len(lens), w, D)
    P.ecokv_prefill_rope(Q, K, shape, rope, None if far is None else pos, Qo, Ko, Qw)
    q, qs = turned(Q, pos, freq, rot, inter, factor, wt[0], 1e-5)
    k, ks = turned(K, pos, freq, rot, inter, factor, wt[1], 1e-5)
    near(Qo, q, qs, dtype)
    near(Ko, k, ks, dtype)
    for s, e in enumerate(cu[1:]):  # the window's rows are the queries' own, bit for bit
        assert torch.equal(Qw[:, :, s], Qo[:, e - w:e].transpose(1, 2))
    # keys alone, the window's queries alone, and both in place give the same bits
    Ko2, Qw2 = out(L, n, Hkv, D), out(L, Hq, len(lens), w, D)
    P.ecokv_prefill_rope(None, K, shape, rope, pos, None, Ko2)
    P.ecokv_prefill_rope(Q, None, shape, rope, pos, Q_win=Qw2)
    assert torch.equal(Ko2, Ko) and torch.equal(Qw2, Qw)
    Qi, Ki = Q.contiguous(), K.contiguous()
    P.ecokv_prefill_rope(Qi, Ki, shape, rope, pos, Qi, Ki)
    assert torch.equal(Qi, Qo) and torch.equal(Ki, Ko)


def test_prefill_rope_long_prompt():
    # more tokens than one round of blocks takes; a norm of one side only
    import paper_2609_06663_amd as P
    L, n, Hq, Hkv, D = 1, 30011, 8, 4, 128
    Q, K, _, freq, wt = make(12, "bf16", L, n, Hq, Hkv, D, 128, True)
    say("30011 tokens, keys normed, queries not")
    Qo, Ko = torch.empty(L, n, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(L, n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    P.ecokv_prefill_rope(Q, K, P.Shape(L, Hq, Hkv, D, 4, [0, n]), P.Rope(128, freq, k_norm=wt[1]), None, Qo, Ko)
    pos = torch.arange(n, device="cuda")
    near(Qo, *turned(Q, pos, freq, 128, False, 1.0, None, 0), "bf16")
    near(Ko, *turned(K, pos, freq, 128, False, 1.0, wt[1], 1e-6), "bf16")


def test_norm_of_zero_and_huge_rows():
    import paper_2609_06663_amd as P
    n, Hq, D = 4, 2, 64
    Q = torch.zeros(1, n, Hq, D, device="cuda")
    Q[0, 1] = 1e18            # squares that float32 still holds
    Q[0, 2, 0, 5] = -3.0      # one element alone
    Q[0, 3] = float("nan")
    w = torch.ones(D, device="cuda")
    out = torch.empty_like(Q)
    P.ecokv_prefill_rope(Q, None, P.Shape(1, Hq, Hq, D, 1, [0, n]), P.Rope(0, q_norm=w, norm_eps=1e-6), None, out)
    assert bool((out[0, 0] == 0).all()) and bool(out[0, 3].isnan().all())
    near(out[:, 1:3], *turned(Q[:, 1:3], torch.zeros(2, device="cuda"), None, 0, False, 1.0, w, 1e-6), "f32")


def pool_of(g, L, pages, Hkv, page, D, dtype):
    return torch.randn((L, pages, Hkv, page, D), generator=g, device="cuda").to(TYPES[dtype])


@pytest.mark.parametrize("dtype,D,Hq,Hkv,rot,inter,norm,L,page", [
    ("bf16", 128, 28, 4, 128, False, False, 1, 16), ("bf16", 128, 32, 8, 64, True, True, 2, 64), ("bf16", 64, 9, 3, 64, False, True, 1, 1),
    ("f32", 128, 2, 2, 128, True, False, 3, 8), ("f32", 64, 8, 4, 16, False, True, 1, 256), ("bf16", 128, 64, 1, 0, False, False, 1, 2)])
@pytest.mark.parametrize("tokens", [[1], [1] * 37, [5, 1, 129, 2, 40]])
def test_append(dtype, D, Hq, Hkv, rot, inter, norm, L, page, tokens):
    import paper_2609_06663_amd as P
    N, n = len(tokens) + 1, sum(tokens)  # the last continuation gets nothing
    say(f"{dtype} D={D} Hq={Hq} Hkv={Hkv} rot={rot} L={L} page={page}: {len(tokens)} continuations, {n} tokens")
    Q, K, V, freq, wt = make(21, dtype, L, n, Hq, Hkv, D, rot, norm)
    g = torch.Generator(device="cuda").manual_seed(22)
    start = [(17 * c) % 50 for c in range(N)]
    per = max((s + t - 1) // page + 1 for s, t in zip(start, tokens + [1]))
    pages = N * per + 5
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(23))[:N * per].view(N, per).int().cuda()
    tk, tv = pool_of(g, L, pages, Hkv, page, D, dtype), pool_of(g, L, pages, Hkv, page, D, dtype)
    conts = torch.tensor([c for c, t in enumerate(tokens) for _ in range(t)], dtype=torch.int32, device="cuda")
    rows = torch.tensor([s + j for s, t in zip(start, tokens) for j in range(t)], dtype=torch.int32, device="cuda")
    pos = rows + 5000 + 7 * conts
    want_k, want_v, written = tk.double(), tv.clone(), torch.zeros(L, pages, Hkv, page, dtype=torch.bool, device="cuda")
    k, ks = turned(K, pos, freq, rot, inter, 1.0, wt[1], 1e-6)
    slack = want_k.abs() * 0
    for t in range(n):
        p, r = int(table[conts[t], rows[t] // page]), int(rows[t] % page)
        want_k[:, p, :, r], want_v[:, p, :, r], slack[:, p, :, r], written[:, p, :, r] = k[:, t], V[:, t], ks[:, t], True
    before = tk.clone()
    tails = P.Tails(tk, tv, table)
    Qd = torch.full((L, Hq, n, D), 7.0, dtype=TYPES[dtype], device="cuda")
    rope = P.Rope(rot, freq, inter, 1.0, *wt)
    shape = P.Shape(L, Hq, Hkv, D, 4, [0, 100])
    P.ecokv_append(Q, K, V, shape, rope, pos, conts if len(set(tokens)) > 1 else None, rows, tails, Qd)
    q, qs = turned(Q, pos, freq, rot, inter, 1.0, wt[0], 1e-6)
    near(Qd, q.transpose(1, 2), qs.transpose(1, 2), dtype)
    near(tk, want_k, slack, dtype)
    assert torch.equal(tv, want_v)
    assert torch.equal(tk[~written], before[~written])
    # without queries the rows are the same
    tk2, tv2 = before.clone(), tv.clone()
    P.ecokv_append(None, K.contiguous(), V.contiguous(), shape, rope, pos, conts, rows, P.Tails(tk2, tv2, table))
    assert torch.equal(tk2, tk) and torch.equal(tv2, tv)


def test_append_leaves_padding_and_bad_pages_alone():
    # rows of -1 and past the table, continuations outside it, pages outside the
    # pool: nothing is written for them (the host test of the same arithmetic is
    # tests/test_shared_plan.py); their queries are rotated like the others'
    import paper_2609_06663_amd as P
    L, Hq, Hkv, D, page, N = 2, 4, 2, 128, 16, 4
    conts = torch.tensor([0, 1, 2, 3, 0, -1, 4, 1, 2], dtype=torch.int32, device="cuda")
    rows = torch.tensor([3, -1, 17, 40, 48, 0, 0, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    n = len(rows)
    table = torch.tensor([[5, 1, 2], [0, 3, 4], [6, 99, 0], [7, 8, -3]], dtype=torch.int32, device="cuda")
    Q, K, V, freq, _ = make(31, "bf16", L, n, Hq, Hkv, D, 128, False)
    g = torch.Generator(device="cuda").manual_seed(32)
    tk, tv = pool_of(g, L, 9, Hkv, page, D, "bf16"), pool_of(g, L, 9, Hkv, page, D, "bf16")
    k0, v0 = tk.clone(), tv.clone()
    Qd = torch.full((L, Hq, n, D), 7.0, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    say("one token in place, eight that go nowhere")
    P.ecokv_append(Q, K, V, P.Shape(L, Hq, Hkv, D, 1, [0, 2]), P.Rope(128, freq), pos, conts, rows, P.Tails(tk, tv, table), Qd)
    q, qs = turned(Q, pos, freq, 128, False, 1.0, None, 0)
    near(Qd, q.transpose(1, 2), qs.transpose(1, 2), "bf16")
    k, ks = turned(K, pos, freq, 128, False, 1.0, None, 0)
    near(tk[:, 5, :, 3], k[:, 0], ks[:, 0], "bf16")
    assert torch.equal(tv[:, 5, :, 3], V[:, 0])
    tk[:, 5, :, 3], tv[:, 5, :, 3] = k0[:, 5, :, 3], v0[:, 5, :, 3]
    assert torch.equal(tk, k0) and torch.equal(tv, v0)


def test_append_into_a_pool_past_32_bits():
    # page 70 000 of 32 KiB per head: byte offsets past 2^32, element offsets past 2^31
    import paper_2609_06663_amd as P
    L, Hq, Hkv, D, page, pages = 1, 4, 2, 128, 128, 70001
    Q, K, V, freq, _ = make(41, "bf16", L, 2, Hq, Hkv, D, 128, False)
    tk, tv = (torch.zeros((L, pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert tk.numel() * 2 > 2 ** 32 and tk.numel() > 2 ** 31
    table = torch.tensor([[pages - 1], [0]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([127, 0], dtype=torch.int32, device="cuda")
    say("the last row of a pool of 4.6 GB")
    P.ecokv_append(Q, K, V, P.Shape(L, Hq, Hkv, D, 1, [0, 2]), P.Rope(128, freq), rows, None, rows, P.Tails(tk, tv, table),
                   torch.empty(L, Hq, 2, D, dtype=torch.bfloat16, device="cuda"))
    k, ks = turned(K, rows, freq, 128, False, 1.0, None, 0)
    near(tk[:, -1, :, 127], k[:, 0], ks[:, 0], "bf16")
    near(tk[:, 0, :, 0], k[:, 1], ks[:, 1], "bf16")
    assert torch.equal(tv[:, -1, :, 127], V[:, 0]) and torch.equal(tv[:, 0, :, 0], V[:, 1])
    assert int(tk.view(torch.int16).count_nonzero()) <= 2 * Hkv * D and int((tv != 0).sum()) <= 2 * Hkv * D


def test_the_binding_refuses_what_does_not_fit():
    import paper_2609_06663_amd as P
    Q, K, V, freq, wt = make(51, "bf16", 1, 6, 4, 2, 128, 128, True)
    s = P.Shape(1, 4, 2, 128, 4, [0, 6])
    Qo, Ko = Q.contiguous(), K.contiguous()
    rope = P.Rope(128, freq)
    with pytest.raises(ValueError, match="shape"):
        P.ecokv_prefill_rope(Q[:, :5], K, s, rope, None, Qo, Ko)
    with pytest.raises(ValueError, match="together"):
        P.ecokv_prefill_rope(Q.transpose(1, 2).contiguous().transpose(1, 2), K, s, rope, None, Qo, Ko)
    with pytest.raises(TypeError, match="K must be bf16"):
        P.ecokv_prefill_rope(Q, K.float(), s, rope, None, Qo, Ko)
    with pytest.raises(ValueError, match="Q_out has"):
        P.ecokv_prefill_rope(Q, K, s, rope, None, Qo[:, :5], Ko)
    with pytest.raises(TypeError, match="q_norm must be bf16"):
        P.ecokv_prefill_rope(Q, K, s, P.Rope(128, freq, q_norm=wt[0].float()), None, Qo, Ko)
    with pytest.raises(ValueError, match="freq has"):
        P.ecokv_prefill_rope(Q, K, s, P.Rope(128, freq[:63]), None, Qo, Ko)
    with pytest.raises(TypeError, match="positions must be int32"):
        P.ecokv_prefill_rope(Q, K, s, rope, torch.arange(6, device="cuda"), Qo, Ko)
    with pytest.raises(ValueError, match="Q_out, Q_win or both"):
        P.ecokv_prefill_rope(Q, K, s, rope, None, None, Ko)
    pool = torch.zeros(1, 4, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(6, 1, dtype=torch.int32, device="cuda")
    i = torch.zeros(6, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="the tails have"):
        P.ecokv_append(Q, K, V, s, rope, i, None, i, P.Tails(pool[:, :, :1].contiguous(), pool[:, :, :1].contiguous(), table), Qo)
    with pytest.raises(TypeError, match="tails' K must be bf16"):
        P.ecokv_append(Q, K, V, s, rope, i, None, i, P.Tails(pool.float(), pool.float(), table), Qo)
    with pytest.raises(ValueError, match="rows has"):
        P.ecokv_append(Q, K, V, s, rope, i, None, i[:5], P.Tails(pool, pool.clone(), table), Qo)
    with pytest.raises(P.EcoKVError):  # K and V of the tails are one
        P.ecokv_append(Q, K, V, s, rope, i, None, i, P.Tails(pool, pool, table), Qo)
    with pytest.raises(P.EcoKVError):  # six tokens, four continuations
        P.ecokv_append(Q, K, V, s, rope, i, None, i, P.Tails(pool, pool.clone(), table[:4]), Qo)
    torch.cuda.synchronize()
    assert bool((pool == 0).all())
