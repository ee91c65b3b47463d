"""ecokv_decode_shared against attention in 64 bits: continuations of shared
prompts over kept rows and paged tails, at the sizes, splits, pages and values
where it can go wrong.

Tolerance.  A logit is a float32 sum of D products in some order: off by at most
(D / 4 + 8) roundings of the sum of their magnitudes, dx = 40 * 2^-24 * max_j
sum_d |q_d k_jd| / sqrt(D).  A weight's relative error is at most 2 dx beside its
normalisation, and the weighted sums and merges add fewer than 64 roundings:
  |O - O64| <= (2 dx + 2^-18) max |V|,  |lse - lse64| <= dx + 2^-20 max(1, |lse64|).
"""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-shared] {msg}", file=sys.stderr, flush=True)


class Case:
    """counts [L][Hkv][B], fan sizes [B], tail counts [N]."""

    def __init__(self, seed, dtype, L, Hq, Hkv, D, counts, fan, tails, page=16, kscale=1.0):
        import paper_2609_06663_amd as P
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        t = TYPES[dtype]
        self.dims = (L, Hq, Hkv, D, len(fan))
        self.fan = [0] + [int(v) for v in np.cumsum(fan)]
        N = self.N = self.fan[-1]
        self.counts = torch.tensor(counts, dtype=torch.int32).view(-1).cuda()
        c = self.counts.long().clamp_min(0)
        self.offsets = (c.cumsum(0) - c).int()
        n = max(1, int(c.sum()))
        self.Kc, self.Vc = (kscale * r(n, D)).to(t), r(n, D).to(t)
        self.Q = r(L, Hq, N, D).to(t)
        self.tail_counts = torch.tensor(tails, dtype=torch.int32, device="cuda")
        self.max_count, self.max_tail = max(0, int(self.counts.max())), max(0, max(tails, default=0))
        per = max(1, -(-self.max_tail // page))
        pages = N * per + 2
        self.table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:N * per].view(N, per).int().cuda()
        self.tk, self.tv = (kscale * r(L, pages, Hkv, page, D)).to(t), r(L, pages, Hkv, page, D).to(t)
        cu = [0]
        for s in range(len(fan)):
            cu.append(cu[-1] + 1000)
        self.shape = P.Shape(L, Hq, Hkv, D, 4, cu)

    def run(self, **kw):
        import paper_2609_06663_amd as P
        L, Hq, _, D, _ = self.dims
        O = torch.full((L, Hq, self.N, D), -7.0, device="cuda")
        lse = torch.full((L, Hq, self.N), -7.0, device="cuda")
        mc, mt = kw.get("max_count", self.max_count), kw.get("max_tail", self.max_tail)
        ws = torch.full((max(256, P.ecokv_decode_shared_workspace_size(self.shape, self.fan, mc, mt)),), 0xFF, dtype=torch.uint8, device="cuda")
        P.ecokv_decode_shared(self.Q, self.Kc, self.Vc, self.shape, self.fan, self.counts, self.offsets, mc,
                              P.Tails(self.tk, self.tv, self.table) if mt else None, self.tail_counts if mt else None, mt, O, lse, ws)
        torch.cuda.synchronize()
        return O, lse

    def rows_of(self, l, h, c):
        _, _, Hkv, D, B = self.dims
        s = next(s for s in range(B) if self.fan[s] <= c < self.fan[s + 1])
        u = (l * Hkv + h) * B + s
        o, n, t, page = int(self.offsets[u]), max(0, int(self.counts[u])), int(self.tail_counts[c]), self.tk.shape[3]
        p = self.table[c, :-(-t // page)].long()
        return [torch.cat([a[o:o + n], b[l, p, h].reshape(-1, D)[:t]]) for a, b in ((self.Kc, self.tk), (self.Vc, self.tv))]

    def check(self, O, lse, skip=()):
        L, Hq, Hkv, D, _ = self.dims
        G = Hq // Hkv
        for l in range(L):
            for h in range(Hkv):
                for c in range(self.N):
                    if c in skip:
                        continue
                    K, V = (x.double() for x in self.rows_of(l, h, c))
                    q = self.Q[l, h * G:(h + 1) * G, c].double()
                    got, gl = O[l, h * G:(h + 1) * G, c], lse[l, h * G:(h + 1) * G, c]
                    if not len(K):
                        assert bool((got == 0).all()) and bool((gl == -float("inf")).all()), (l, h, c)
                        continue
                    x = q @ K.t() / D ** 0.5
                    dx = 40 * 2.0 ** -24 * float((q.abs() @ K.abs().t()).nan_to_num(0, 0, 0).max()) / D ** 0.5
                    ref, rl = x.softmax(1) @ V, x.logsumexp(1)
                    err = float((got.double() - ref).abs().max())
                    assert err <= (2 * dx + 2.0 ** -18) * float(V.abs().max()), (l, h, c, len(K), err, dx)
                    assert bool(((gl.double() - rl).abs() <= dx + 2.0 ** -20 * rl.abs().clamp_min(1)).all()), (l, h, c)


SHAPES = [  # dtype, D, L, Hq, Hkv, counts (per unit), fan, tails, page
    ("bf16", 128, 1, 28, 4, [6553], [8], [200, 1, 0, 64, 65, 128, 199, 37], 64),
    ("bf16", 128, 1, 28, 4, [700, 33], [3, 2], [5, 16, 17, 0, 129], 16),
    ("bf16", 128, 2, 32, 8, [1500, 1, 64, 0, 129], [5, 1, 12, 0, 3], [7 * i % 50 for i in range(21)], 8),
    ("bf16", 64, 1, 8, 8, [2049], [20], [100] * 20, 1),
    ("bf16", 64, 3, 6, 2, [40, 257], [1, 1], [300, 2], 128),
    ("bf16", 128, 1, 64, 1, [1000], [2], [40, 33], 16),
    ("bf16", 128, 1, 17, 1, [515], [40], [i for i in range(40)], 4),
    ("bf16", 128, 1, 4, 2, [2000], [64], [11 * i % 400 for i in range(64)], 32),
    ("bf16", 128, 1, 28, 4, [1030], [37], [5] * 37, 16),
    ("f32", 128, 1, 8, 4, [300, 20], [3, 2], [50, 0, 1, 17, 16], 16),
    ("f32", 128, 1, 2, 2, [128], [2], [5, 4], 16),
    ("f32", 64, 2, 12, 4, [1, 515], [9, 1], [3 * i for i in range(10)], 2),
    ("f32", 64, 1, 40, 1, [900], [3], [200, 100, 1], 64),
    ("f32", 128, 1, 28, 4, [611], [21], [9 * i % 70 for i in range(21)], 16),
]


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: f"{c[0]}-D{c[1]}-L{c[2]}-{c[3]}q{c[4]}kv-{c[5]}-{c[6]}-p{c[8]}")
@pytest.mark.parametrize("kscale", [1.0, 8.0])
def test_shared(case, kscale):
    dtype, D, L, Hq, Hkv, counts, fan, tails, page = case
    say(f"{case[:7]} page {page} keys x {kscale}")
    # the heads of a prompt keep different numbers of rows
    per = [[[max(0, n - 13 * ((3 * h + l) % 4)) if n > 60 else n for n in counts] for h in range(Hkv)] for l in range(L)]
    c = Case(7, dtype, L, Hq, Hkv, D, per, fan, tails, page, kscale)
    O, lse = c.run()
    c.check(O, lse)
    # bounds above the counts split the rows otherwise
    top = c.table.shape[1] * page
    O2, lse2 = c.run(max_count=4 * c.max_count + 900, max_tail=top)
    c.check(O2, lse2)
    # and a second call gives the same bits
    O3, lse3 = c.run()
    assert torch.equal(O, O3) and torch.equal(lse, lse3)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: f"{c[0]}-D{c[1]}-L{c[2]}-{c[3]}q{c[4]}kv-{c[5]}-{c[6]}-p{c[8]}")
def test_shared_as_in_large_calls(case):
    # a bound of 3 million kept rows: split like a call that reads gigabytes, with
    # blocks of as many query rows as the largest prompt fills
    dtype, D, L, Hq, Hkv, counts, fan, tails, page = case
    say(f"{case[:7]} page {page}, split for 3 million rows")
    c = Case(20, dtype, L, Hq, Hkv, D, [[counts] * Hkv] * L, fan, tails, page)
    O, lse = c.run(max_count=3_000_000)
    c.check(O, lse)
    O2, lse2 = c.run(max_count=3_000_000)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_rows_of_weight_zero_in_large_calls(dtype, D):
    # the same with dead rows at a part's ends, and NaN in one unit
    c = Case(21, dtype, 1, 8, 2, D, [[[1400], [600]]], [20], [50, 0] * 10, 16)
    c.Q[..., 0] = 1.0
    c.Kc[:300, 0] = -float("inf")
    c.Kc[1350:1400, 0] = -float("inf")
    c.Kc[1700, 3] = float("nan")
    say(f"{dtype} D={D}: rows of weight zero, split for 3 million rows")
    O, lse = c.run(max_count=3_000_000)
    assert bool(O[:, 4:].isnan().all()) and bool(lse[:, 4:].isnan().all())
    for k in range(20):
        K, V = (x.double() for x in c.rows_of(0, 0, k))
        q = c.Q[0, :4, k].double()
        dead = K[:, 0] == -float("inf")
        x = (q @ K.masked_fill(dead[:, None], 0).t() / D ** 0.5).masked_fill(dead, -float("inf"))
        assert float((O[0, :4, k].double() - x.softmax(1) @ V).abs().max()) <= 1e-4 * float(V.abs().max()), k
        assert bool(((lse[0, :4, k].double() - x.logsumexp(1)).abs() <= 1e-4).all()), k


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_prompt_alone_and_tail_alone(dtype, D):
    c = Case(8, dtype, 1, 14, 2, D, [[[333, 129], [400, 1]]], [3, 2], [40, 1, 77, 0, 16], 16)
    say(f"{dtype} D={D}: without tails, without prompts")
    full = c.tail_counts.clone()
    c.tail_counts.zero_()
    O, lse = c.run()                       # empty tails
    O1, lse1 = c.run(max_tail=0)           # no tails at all
    c.check(O, lse)
    c.check(O1, lse1)
    c.tail_counts.copy_(full)
    c.counts.zero_()
    O, lse = c.run()                       # prompts of which nothing was kept
    c.check(O, lse)
    O1, lse1 = c.run(max_count=0)
    c.check(O1, lse1)


@pytest.mark.parametrize("dtype,D,N", [("bf16", 128, 5), ("f32", 64, 1)])
def test_neither_prompts_nor_tails(dtype, D, N):
    # both bounds 0: the workspace has no places, and none may be read
    import paper_2609_06663_amd as P
    c = Case(19, dtype, 1, 8, 2, D, [[[0], [0]]], [N], [0] * N, 16)
    say(f"{dtype} D={D}: no rows at all")
    assert P.ecokv_decode_shared_workspace_size(c.shape, c.fan, 0, 0) == 0
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        O, lse = torch.full((1, 8, N, D), -7.0, device="cuda"), torch.full((1, 8, N), -7.0, device="cuda")
        P.ecokv_decode_shared(c.Q, None, None, c.shape, c.fan, None, None, 0, None, None, 0, O, lse, ws)
        torch.cuda.synchronize()
        assert bool((O == 0).all()) and bool((lse == -float("inf")).all())


def test_one_continuation_each_is_plain_decode():
    import paper_2609_06663_amd as P
    c = Case(9, "bf16", 2, 28, 4, 128, [[[900, 64, 2000]] * 4] * 2, [1, 1, 1], [0, 0, 0], 16)
    O, lse = c.run(max_tail=0)
    O2, lse2 = torch.empty_like(O), torch.empty_like(lse)
    P.ecokv_decode(c.Q, c.Kc, c.Vc, c.shape, c.counts, c.offsets, 2000, O2, lse2)
    # each within a few 2^-24 of the exact sums: the logits' error, twice
    say("against ecokv_decode")
    assert float((O - O2).abs().max()) <= 2.0 ** -16 * float(c.Vc.abs().max())
    assert float((lse - lse2).abs().max()) <= 2.0 ** -16 * 8


def test_counts_out_of_their_bounds_are_nan():
    c = Case(10, "f32", 1, 4, 2, 64, [[[100, 90], [300, 20]]], [2, 3], [10, 20, 30, 5, 40], 16)
    say("counts below 0 and above their bounds")
    c.counts[1] = -1                       # KV head 0, prompt 1: continuations 2..4
    O, lse = c.run(max_count=200, max_tail=30)   # KV head 1, prompt 0: 300 rows; continuation 4: 40 rows
    bad = torch.zeros(1, 4, 5, dtype=torch.bool, device="cuda")
    bad[:, :2, 2:], bad[:, 2:, :2], bad[:, :, 4] = True, True, True
    assert bool(O[bad].isnan().all()) and bool(lse[bad].isnan().all())
    assert bool(O[~bad].isfinite().all()) and bool(lse[~bad].isfinite().all())
    c.tail_counts[0] = -7
    O, lse = c.run(max_count=300, max_tail=40)
    assert bool(O[:, :, 0].isnan().all()) and bool(O[:, 2:, 1:].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_outside_the_pool_give_nan(dtype):
    # (the arithmetic that finds them is tested on the host, tests/test_shared_plan.py)
    c = Case(11, dtype, 1, 28, 4, 128, [[[300]] * 4], [5], [70, 70, 70, 70, 30], 16)
    c.table[1, 4], c.table[2, 0], c.table[4, 2] = c.tk.shape[1], -1, 2 ** 31 - 1  # (the last one's page is not read: 30 rows)
    say(f"{dtype}: pages outside the pool")
    O, lse = c.run()
    assert bool(O[:, :, 1:3].isnan().all()) and bool(lse[:, :, 1:3].isnan().all())
    c.check(O, lse, skip=(1, 2))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_rows_of_weight_zero_and_nan(dtype, D):
    c = Case(12, dtype, 1, 8, 2, D, [[[700], [200]]], [4], [50, 0, 33, 129], 16)
    c.Q[..., 0] = 1.0
    # logits of -inf: the first rows, whole tiles, a whole unit's first wave, a whole tail
    c.Kc[:40, 0] = -float("inf")
    c.Kc[128:300, 0] = -float("inf")
    c.Kc[700:860, 0] = -float("inf")
    c.tk[:, c.table[2].long(), :, :, 0] = -float("inf")
    say(f"{dtype} D={D}: rows of weight zero")
    O, lse = c.run()
    for h in range(2):
        for k in range(4):
            K, V = (x.double() for x in c.rows_of(0, h, k))
            q = c.Q[0, 4 * h:4 * h + 4, k].double()
            dead = K[:, 0] == -float("inf")
            x = (q @ K.masked_fill(dead[:, None], 0).t() / D ** 0.5).masked_fill(dead, -float("inf"))
            assert float((O[0, 4 * h:4 * h + 4, k].double() - x.softmax(1) @ V).abs().max()) <= 1e-4 * float(V.abs().max()), (h, k)
            assert bool(((lse[0, 4 * h:4 * h + 4, k].double() - x.logsumexp(1)).abs() <= 1e-4).all())
    # every row dead: nothing is attended
    c.Kc[..., 0] = -float("inf")
    c.tk[..., 0] = -float("inf")
    O, lse = c.run()
    assert bool((O == 0).all()) and bool((lse == -float("inf")).all())
    # NaN in a row of unit 1, and in the tail of continuation 3
    c = Case(13, dtype, 1, 8, 2, D, [[[700], [200]]], [4], [50, 0, 33, 129], 16)
    c.Kc[850, 3] = float("nan")
    c.tk[:, c.table[3, 8].long(), :, 0, 5] = float("nan")   # row 128
    O, lse = c.run()
    bad = torch.zeros(1, 8, 4, dtype=torch.bool, device="cuda")
    bad[:, 4:], bad[:, :, 3] = True, True
    assert bool(O[bad].isnan().all()) and bool(O[~bad].isfinite().all()) and bool(lse[~bad].isfinite().all())


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_what_lies_behind_the_rows_is_not_attended(dtype, D):
    # infinities and NaN after a unit's rows, after a tail's and in pages of nobody
    c = Case(14, dtype, 1, 4, 2, D, [[[100], [37]]], [3], [50, 1, 33], 16)
    for t in (c.Kc, c.Vc):
        t.resize_(137 + 64, D)[137:] = float("inf")
    own = torch.zeros(c.tk.shape[1], c.tk.shape[3], dtype=torch.bool, device="cuda")
    for k, n in enumerate([50, 1, 33]):
        for r in range(n):
            own[c.table[k, r // 16].long(), r % 16] = True
    c.tk[0].transpose(1, 2)[~own] = float("nan")
    c.tv[0].transpose(1, 2)[~own] = float("inf")
    say(f"{dtype} D={D}: poison behind the rows")
    c.check(*c.run())


def test_a_cache_past_32_bits():
    # kept rows and pages whose byte offsets pass 2^32 (element offsets 2^31)
    import paper_2609_06663_amd as P
    D, n = 128, 17_000_000
    Kc, Vc = (torch.empty(n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Case(15, "bf16", 1, 4, 1, D, [[[300]]], [2], [100, 70], 128)
    Kc[n - 300:], Vc[n - 300:] = c.Kc, c.Vc
    pages = 140_001
    tk, tv = (torch.empty((1, pages, 1, 128, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert Kc.numel() > 2 ** 31 and tk.numel() > 2 ** 31
    for k in range(2):
        tk[0, pages - 1 - k], tv[0, pages - 1 - k] = c.tk[0, c.table[k, 0].long()], c.tv[0, c.table[k, 0].long()]
    say("the end of caches of 4.4 and 4.6 GB")
    table = torch.tensor([[pages - 1], [pages - 2]], dtype=torch.int32, device="cuda")
    O, lse = torch.empty(1, 4, 2, D, device="cuda"), torch.empty(1, 4, 2, device="cuda")
    P.ecokv_decode_shared(c.Q, Kc, Vc, c.shape, [0, 2], c.counts, c.offsets + (n - 300), 300, P.Tails(tk, tv, table), c.tail_counts, 100, O, lse)
    torch.cuda.synchronize()
    c.check(O, lse)


def test_pages_that_two_continuations_share():
    # a fork: continuations 0 and 1 read the same first two pages
    c = Case(16, "bf16", 1, 8, 2, 128, [[[64], [64]]], [3], [40, 45, 20], 16)
    c.table[1, :2] = c.table[0, :2]
    c.check(*c.run())


def test_many_query_rows():
    # 1.3 million query rows: more merges than one grid dimension holds
    import paper_2609_06663_amd as P
    L, Hq, Hkv, D, N = 20, 64, 1, 64, 1030
    say(f"{L * Hq * N} query rows")
    Q = torch.zeros(L, Hq, N, D, dtype=torch.bfloat16, device="cuda")
    Kc, Vc = (torch.arange(D, dtype=torch.bfloat16, device="cuda").repeat(3, 1) + x for x in (1, 2))
    n = torch.full((L,), 3, dtype=torch.int32, device="cuda")
    O, lse = torch.full((L, Hq, N, D), -7.0, device="cuda"), torch.full((L, Hq, N), -7.0, device="cuda")
    P.ecokv_decode_shared(Q, Kc, Vc, P.Shape(L, Hq, Hkv, D, 1, [0, 9]), [0, N], n, torch.zeros_like(n), 3, None, None, 0, O, lse)
    assert bool(((O - Vc[0].float()).abs() <= 2.0 ** -20 * 70).all()) and bool(((lse - np.log(3)).abs() <= 1e-6).all())


def test_the_binding_refuses_what_does_not_fit():
    import paper_2609_06663_amd as P
    c = Case(17, "bf16", 1, 4, 2, 64, [[[30], [40]]], [2], [5, 6], 16)
    O, lse = torch.empty(1, 4, 2, 64, device="cuda"), torch.empty(1, 4, 2, device="cuda")
    t = P.Tails(c.tk, c.tv, c.table)
    call = lambda **kw: P.ecokv_decode_shared(*[kw.get(n, v) for n, v in dict(Q=c.Q, K=c.Kc, V=c.Vc, shape=c.shape, fan=c.fan, n=c.counts, o=c.offsets,
                                                                               mc=40, t=t, tc=c.tail_counts, mt=6, O=O, lse=lse, ws=None).items()])
    call()
    for kw, err in ((dict(Q=c.Q[:, :3]), ValueError), (dict(K=c.Kc.float()), TypeError), (dict(V=c.Vc[:-1]), ValueError), (dict(n=c.counts.long()), TypeError),
                    (dict(o=c.offsets[:1]), ValueError), (dict(t=None), ValueError), (dict(tc=None), ValueError), (dict(tc=c.tail_counts[:1]), ValueError),
                    (dict(O=O.bfloat16()), TypeError), (dict(O=O[:, :3]), ValueError), (dict(lse=lse[:, :3]), ValueError), (dict(K=None), ValueError),
                    (dict(ws=torch.empty(256, dtype=torch.uint8, device="cuda")), P.EcoKVError), (dict(ws=torch.empty(256, device="cuda")), TypeError), (dict(fan=[0, 1]), P.EcoKVError), (dict(mt=17), P.EcoKVError)):
        with pytest.raises(err):
            call(**kw)
