"""ecokv_decode_shared where a call is large: query tiles of two and four waves
over parts of many tiles (tests/test_gpu_shared.py reaches these tiles with one or
two), and grids past one dimension.  The splits that the sizes are there for are
checked on the host, tests/test_shared_plan_wide.py.

Tolerance: that of tests/test_gpu_shared.py, whose 64 roundings of sums hold for
short parts; here a wave adds up to R rows to one sum, bf16 values in three
products each and the weights' sum besides, less than 4 R roundings.  Each is of
at most 2^-24 of sum_j w_j |v_j|, as is what the weights' errors make:
  |O - O64| <= (2 dx + 2^-18 + 4 R 2^-24) sum_j w_j |v_j|,
  |lse - lse64| <= dx + R 2^-24 + 2^-20 max(1, |lse64|).
"""
import sys

import pytest
import torch
from shared_sizes import GRID_MERGE, GRID_PROMPTS, GRID_TAILS, SHARED_BOUND, SHARED_BUDGET, SHARED_WAVE, TAIL, WIDE, kept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-shared-wide] {msg}", file=sys.stderr, flush=True)


def check_rows(q, K, V, O, lse, rows, where):
    """Query rows q [G][D] over K and V in 64 bits."""
    q, K, V = q.double(), K.double(), V.double()
    x = q @ K.t() / q.shape[-1] ** 0.5
    dx = 40 * 2.0 ** -24 * float((q.abs() @ K.abs().t()).max()) / q.shape[-1] ** 0.5
    w = x.softmax(1)
    err = (O.double() - w @ V).abs()
    assert bool((err <= (2 * dx + 2.0 ** -18 + rows * 2.0 ** -22) * (w @ V.abs())).all()), (where, len(K), float(err.max()))
    rl = x.logsumexp(1)
    assert bool(((lse.double() - rl).abs() <= dx + rows * 2.0 ** -24 + 2.0 ** -20 * rl.abs().clamp_min(1)).all()), where


@pytest.mark.parametrize("case", WIDE, ids=str)
def test_wide_tiles_over_long_parts(case):
    import paper_2609_06663_amd as P
    from test_gpu_shared import Case
    dtype, D, L, Hq, Hkv, counts, fan, _, wave = case
    say(f"{case}")
    N = sum(fan)
    c = Case(70, dtype, L, Hq, Hkv, D, kept(case), fan, [(13 * i + 70) % (TAIL + 1) for i in range(N)], 16)
    assert c.max_count == max(counts) and c.max_tail == TAIL
    O, lse = c.run()
    # twelve (layer, head)s against 64 bits, the longest and the single rows among them
    pairs = {(0, 0), (1, 0), (L - 1, Hkv - 1)} | {(5 * i % L, i % Hkv) for i in range(1, 10)}
    G = Hq // Hkv
    for l, h in sorted(pairs):
        for k in range(N):
            at = l, slice(h * G, h * G + G), k
            check_rows(c.Q[at], *c.rows_of(l, h, k), O[at], lse[at], wave, (l, h, k))
    # and all of them against calls of one layer, split otherwise (in no longer sums)
    dx = 40 * 2.0 ** -24 * float(c.Q.float().norm(dim=-1).max()) * float(torch.cat([c.Kc, c.tk.view(-1, D)]).float().norm(dim=-1).max()) / D ** 0.5
    most = float(torch.maximum(c.Vc.abs().max(), c.tv.abs().max()))
    one, u = P.Shape(1, Hq, Hkv, D, 4, c.shape.cu_seqlens), Hkv * len(fan)
    for l in range(L):
        Ol, ll = torch.empty_like(O[l]), torch.empty_like(lse[l])
        P.ecokv_decode_shared(c.Q[l], c.Kc, c.Vc, one, c.fan, c.counts[l * u:(l + 1) * u], c.offsets[l * u:(l + 1) * u], c.max_count,
                              P.Tails(c.tk[l:l + 1], c.tv[l:l + 1], c.table), c.tail_counts, TAIL, Ol, ll)
        assert bool(((Ol - O[l]).abs() <= 2 * (2 * dx + 2.0 ** -18 + wave * 2.0 ** -22) * most).all()), l
        assert bool(((ll - lse[l]).abs() <= 2 * (dx + wave * 2.0 ** -24 + 2.0 ** -20 * ll.abs().clamp_min(1))).all()), l
    # and the same bits again
    O2, lse2 = c.run()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


def one_row_each(Q, K, V, O, lse):
    """Outputs of query rows Q [..., D] that attend one row each, K and V: the value itself, and the logit."""
    D = Q.shape[-1]
    assert bool(((O - V.float()).abs() <= 2.0 ** -20 * V.float().abs()).all())
    q, k = Q.double(), K.double()
    bound = 40 * 2.0 ** -24 * (q.abs() * k.abs()).sum(-1) / D ** 0.5
    x = (q * k).sum(-1) / D ** 0.5
    assert bool(((lse.double() - x).abs() <= bound + 2.0 ** -20 * x.abs().clamp_min(1)).all())


def test_more_tails_than_one_dimension_holds():
    # every query row has a value of its own, so that one in another's place shows
    import paper_2609_06663_amd as P
    L, Hq, Hkv, D, N, _, mt = GRID_TAILS
    say(f"{L * Hkv * N} tails of one row")
    g = torch.Generator(device="cuda").manual_seed(71)
    r = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, tk, tv = r(L, Hq, N, D), r(L, N, Hkv, 1, D), r(L, N, Hkv, 1, D)
    table = torch.randperm(N, generator=torch.Generator().manual_seed(72)).int().cuda().view(N, 1)
    ones = torch.ones(N, dtype=torch.int32, device="cuda")
    O, lse = torch.full((L, Hq, N, D), -7.0, device="cuda"), torch.full((L, Hq, N), -7.0, device="cuda")
    P.ecokv_decode_shared(Q, None, None, P.Shape(L, Hq, Hkv, D, 4, [0, 10]), [0, N], None, None, 0, P.Tails(tk, tv, table), ones, mt, O, lse)
    torch.cuda.synchronize()
    at = table.view(-1).long()
    for l in range(L):
        for h in range(Hkv):
            one_row_each(Q[l, h], tk[l, at, h, 0], tv[l, at, h, 0], O[l, h], lse[l, h])


@pytest.mark.parametrize("size", [GRID_PROMPTS, GRID_MERGE], ids=str)
def test_more_prompts_than_one_dimension_holds(size):
    import paper_2609_06663_amd as P
    L, Hq, Hkv, D, B, mc, _ = size
    units = L * Hkv * B
    say(f"{units} units of one row, bound {mc}")
    g = torch.Generator(device="cuda").manual_seed(73)
    r = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    Q, Kc, Vc = r(L, Hq, B, D), r(units, D), r(units, D)
    offsets = torch.randperm(units, generator=torch.Generator().manual_seed(74)).int().cuda()
    ones = torch.ones(units, dtype=torch.int32, device="cuda")
    O, lse = torch.full((L, Hq, B, D), -7.0, device="cuda"), torch.full((L, Hq, B), -7.0, device="cuda")
    P.ecokv_decode_shared(Q, Kc, Vc, P.Shape(L, Hq, Hkv, D, 4, [10 * s for s in range(B + 1)]), list(range(B + 1)), ones, offsets, mc, None, None, 0, O, lse)
    torch.cuda.synchronize()
    at = offsets.view(L, Hkv, B).long()
    for l in range(L):
        one_row_each(Q[l], Kc[at[l]], Vc[at[l]], O[l], lse[l])


def test_generation_from_prompts_whose_heads_share_a_budget():
    # the most that one head of a layer may keep is four times what a head keeps: the
    # bound alone makes the call a wide one
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    from test_gpu_generate import Model
    L, Hq, Hkv, D, G, N = 7, 28, 4, 128, 7, 16
    m = Model(75, "bf16", L, Hq, Hkv, D, 4, [8000])
    ep = m.prefill([SHARED_BUDGET], P.LAYER_FLAT)
    co = Continuations(ep, [N], 3, m.rope, 2)
    assert co.max_count == SHARED_BOUND and int(ep.counts.sum()) == L * Hkv * SHARED_BUDGET
    counts, offsets = ep.counts.tolist(), ep.offsets.tolist()
    for step in range(3):
        Q, K, V = m.project(N)
        co.step(Q, K, V)
        say(f"token {step}: {min(counts)} to {max(counts)} rows a head")
        for l in range(L):
            for h in range(Hkv):
                o, n = offsets[l * Hkv + h], counts[l * Hkv + h]
                for k in (0, 5, N - 1):
                    pages = co.tails.table[k].long()
                    rows = [torch.cat([a[o:o + n], t[l, pages, h].reshape(-1, D)[:step + 1]]) for a, t in ((ep.Kc, co.tails.K), (ep.Vc, co.tails.V))]
                    at = l, slice(h * G, h * G + G), k
                    check_rows(co.Q_dec[at], *rows, co.O[at], co.lse[at], SHARED_WAVE, (l, h, k))
        co.advance()
