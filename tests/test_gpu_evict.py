"""ecokv_accumulate against weights in 64 bits, ecokv_evict and ecokv_evict_tails
against the rows that a sort keeps, at the sizes, paths, pages and masses where they
can go wrong.

Tolerance of a mass.  dx bounds a logit's error (cache_cases.logit_error).  A weight's
exponent t = x - lse is off by dx and a few roundings of itself, so the weight by at
most 2 dx + 2^-20 + 2^-22 |t| of itself (exp2 and the product with log2 e: 2^-22 |t| and
2 units); a row's sum of n weights adds n + 4 roundings of itself, decay twice one:
  |out - out64| <= sum_i w_i (2 dx + 2^-20 + 2^-22 |t_i| + (n + 4) 2^-24)
                   + 2^-22 decay in + n 2^-126.
Evictions are exact.
"""
import random
import sys

import pytest
import torch

from cache_cases import Cache, logit_error

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-evict] {msg}", file=sys.stderr, flush=True)


class Masses(Cache):
    """A cache after a step: queries, their log-sum-exps, masses.  nodes = 0: one query of each continuation."""

    def __init__(self, seed, dtype, L, Hq, Hkv, D, counts, fan, tails, nodes=0, accepted=None, **kw):
        super().__init__(seed, dtype, L, Hq, Hkv, D, counts, fan, tails, **kw)
        M = self.M = max(1, nodes)
        rng, N = random.Random(seed), self.N
        self.acc = [1] * N if not nodes else accepted or [min(max(0, tails[c]), [0, M, rng.randint(0, M), 1][c % 4]) for c in range(N)]
        self.path = [[0]] * N if not nodes else [sorted(rng.sample(range(M), a)) + [0] * (M - a) for a in self.acc]
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda").contiguous()  # noqa: E731
        self.path_t, self.acc_t = (i32(self.path).view(N, M), i32(self.acc)) if nodes else (None, None)
        r = lambda *s: torch.randn(s, generator=self.g, device="cuda")  # noqa: E731
        self.Q = r(L, Hq, N * M, D).to(self.type)
        self.lse = 3 + r(L, Hq, N * M)
        self.mass, self.tail_mass = r(self.Kc.shape[0]).exp(), r(*self.tk.shape[:-1]).exp()

    def run(self, decay=1.0, out=None, stream=None, **kw):
        import paper_2609_06663_amd as P
        mc, mt = kw.get("max_count", self.max_count), kw.get("max_tail", self.max_tail)
        mo, to = out or (torch.full_like(self.mass, -7.0), torch.full_like(self.tail_mass, -7.0))
        P.ecokv_accumulate(self.Q, self.lse, self.Kc, self.shape, self.fan, self.counts, self.offsets, mc, self.tails, self.tail_counts, mt,
                           self.mass, self.tail_mass, self.path_t, self.acc_t, decay, mo, to, stream)
        torch.cuda.synchronize()
        return mo, to

    def check(self, mo, to, decay, skip_units=(), skip_conts=()):
        L, Hq, Hkv, D, B = self.dims
        G, M = Hq // Hkv, self.M
        untouched, tail_untouched = torch.ones_like(mo, dtype=torch.bool), torch.ones_like(to, dtype=torch.bool)

        def weights(K, q, lse, hidden=None):
            x = q @ K.t() / D ** 0.5 - lse[:, None]
            if hidden is not None:
                x = x.masked_fill(hidden, -float("inf"))
            w = torch.where(torch.isneginf(lse)[:, None], 0.0, x.exp())
            tol = 2 * logit_error(q, K, D) + 2.0 ** -20 + 2.0 ** -22 * x.abs().nan_to_num(0, 0, 0) + (len(q) + 4) * 2.0 ** -24
            return w.sum(0), (w * tol).sum(0) + len(q) * 2.0 ** -126

        for l in range(L):
            for h in range(Hkv):
                heads = slice(h * G, (h + 1) * G)
                pick = lambda c: [c * M + v for v in self.path[c][:self.acc[c]]]  # noqa: E731
                for s in range(B):
                    u = (l * Hkv + h) * B + s
                    o, n = int(self.offsets[u]), int(self.counts[u])
                    if u in skip_units or n <= 0:
                        continue
                    at = [i for c in range(self.fan[s], self.fan[s + 1]) for i in pick(c)]
                    q, z = self.Q[l, heads, at].double().reshape(-1, D), self.lse[l, heads, at].double().reshape(-1)
                    w, tol = weights(self.Kc[o:o + n].double(), q, z)
                    before = decay * self.mass[o:o + n].double()
                    err = (mo[o:o + n].double() - w - before).abs()
                    assert bool((err <= tol + 2.0 ** -22 * before).all()), (l, h, s, float((err - tol).max()))
                    untouched[o:o + n] = False
                for c in range(self.N):
                    n, a = int(self.tail_counts[c]), self.acc[c]
                    if c in skip_conts or n <= 0:
                        continue
                    p, r = self.tail_index(c, list(range(n)))
                    q, z = self.Q[l, heads, pick(c)].double(), self.lse[l, heads, pick(c)].double()
                    sees = torch.arange(n, device="cuda") <= torch.arange(n - a, n, device="cuda")[:, None]
                    hidden = ~sees[None].expand(G, -1, -1).reshape(G * a, n)
                    w, tol = weights(self.tk[l, p, h, r].double(), q.reshape(-1, D), z.reshape(-1), hidden)
                    before = decay * self.tail_mass[l, p, h, r].double()
                    before[n - a:] = 0
                    err = (to[l, p, h, r].double() - w - before).abs()
                    assert bool((err <= tol + 2.0 ** -22 * before).all()), (l, h, c, float((err - tol).max()))
                    tail_untouched[l, p, h, r] = False
        return untouched, tail_untouched


SHAPES = [  # dtype, D, L, Hq, Hkv, counts, fan, tails, nodes (0: one query), page
    ("bf16", 128, 1, 28, 4, [6553], [8], [200, 1, 7, 64, 65, 128, 199, 37], 0, 64),
    ("bf16", 128, 2, 32, 8, [1500, 1, 64, 0, 129], [5, 1, 4, 0, 3], [1 + 7 * i % 50 for i in range(13)], 0, 8),
    ("bf16", 64, 1, 8, 8, [2049], [20], [100] * 20, 0, 1),
    ("bf16", 128, 1, 17, 1, [515], [70], [i + 1 for i in range(70)], 0, 4),
    ("bf16", 128, 1, 28, 4, [700, 33], [3, 2], [64, 70, 600, 65, 129], 64, 16),
    ("bf16", 64, 2, 6, 2, [40, 257], [1, 66], [300] + [9 + i for i in range(66)], 9, 128),
    ("bf16", 128, 28, 28, 4, [1000], [4], [500, 300, 1000, 9], 8, 64),
    ("f32", 128, 1, 8, 4, [300, 20], [3, 2], [50, 1, 1, 17, 16], 0, 16),
    ("f32", 64, 2, 12, 4, [1, 515], [9, 1], [3 * i + 8 for i in range(10)], 7, 2),
    ("f32", 128, 20, 2, 2, [3000, 4000], [2, 2], [5, 400, 800, 1], 0, 16),
    ("bf16", 128, 1, 1, 1, [1], [1], [1], 0, 16),
]
IDS = dict(ids=lambda c: f"{c[0]}-D{c[1]}-L{c[2]}-{c[3]}q{c[4]}kv-{c[5]}-{c[6]}-m{c[8]}-p{c[9]}")


def ragged(counts, L, Hkv):
    return [[[max(0, n - 13 * ((3 * h + l) % 4)) if n > 60 else n for n in counts] for h in range(Hkv)] for l in range(L)]


@pytest.mark.parametrize("case", SHAPES, **IDS)
def test_accumulate(case):
    dtype, D, L, Hq, Hkv, counts, fan, tails, nodes, page = case
    say(f"{case[:9]} page {page}")
    t = Masses(7, dtype, L, Hq, Hkv, D, ragged(counts, L, Hkv), fan, tails, nodes, page=page)
    mo, to = t.run(0.75)
    a, b = t.check(mo, to, 0.75)
    assert bool((mo[a] == -7).all()) and bool((to[b] == -7).all())
    # bounds above the counts, and in place: the same bits
    m, tm = t.mass.clone(), t.tail_mass.clone()
    t.run(0.75, (t.mass, t.tail_mass), max_count=3 * t.max_count + 500, max_tail=t.table.shape[1] * page)
    assert torch.equal(t.mass[~a], mo[~a]) and torch.equal(t.tail_mass[~b], to[~b])
    assert torch.equal(t.mass[a], m[a]) and torch.equal(t.tail_mass[b], tm[b])


def test_accumulate_after_attention():
    """The log-sum-exps that attention left: every query's weights add up to 1."""
    import paper_2609_06663_amd as P
    say("weights add up to 1")
    t = Masses(8, "bf16", 2, 8, 2, 128, [[[900], [800]], [[700], [901]]], [3], [40, 1, 129])
    O, lse = torch.empty((2, 8, 3, 128), device="cuda"), torch.empty((2, 8, 3), device="cuda")
    P.ecokv_decode_shared(t.Q, t.Kc, t.Vc, t.shape, t.fan, t.counts, t.offsets, t.max_count, t.tails, t.tail_counts, t.max_tail, O, lse)
    t.lse = lse
    mo, to = t.run(0.0)
    for l in range(2):
        for h in range(2):
            total = float(mo[t.kept(l, h, 0)].double().sum())
            for c in range(3):
                p, r = t.tail_index(c, list(range(int(t.tail_counts[c]))))
                total += float(to[l, p, h, r].double().sum())
            assert abs(total - 12) <= 12 * 2.0 ** -14  # (3 queries of 4 heads; each lse is off by less than 2^-15)


def test_accumulate_edges():
    """Counts out of their bounds, tail rows without a page, queries without a row, paths out of range, -inf and NaN logits."""
    say("accumulate, edges")
    t = Masses(9, "f32", 1, 4, 2, 64, [[[90, 50, 30], [80, 40, 20]]], [2, 2, 2], [40, 41, 90, 43, 17, 30], 5, page=8)
    t.counts[1], t.counts[3] = t.max_count + 1, -1     # prompt 1 of head 0, prompt 0 of head 1
    t.tail_counts[0] = -1
    t.table[4, 1] = t.tk.shape[1]
    t.lse[0, 0, 3 * 5:4 * 5] = -float("inf")            # queries of continuation 3 that saw no row
    mo, to = t.run(0.5, max_tail=60)                    # continuation 2 has 90 rows
    tab = t.table.clone()
    t.table[4, 1] = 0
    a, b = t.check(mo, to, 0.5, skip_units=(1, 3), skip_conts=(0, 2, 4))
    assert bool((mo[a] == -7).all())
    t.table.copy_(tab)
    # continuation 4: rows 8 .. 15 have no page, the others are there
    p, r = t.tail_index(4, [0, 7, 16])
    assert bool((to[0, p, :, r] != -7).all())
    # paths out of range add nothing
    t2 = Masses(9, "f32", 1, 4, 2, 64, [[[90], [80]]], [2], [40, 41], 5, page=8, accepted=[2, 3])
    t2.path_t[0, 0], t2.path_t[1, 2] = -1, 5
    mo, _ = t2.run(0.0, max_tail=0)
    t2.path, t2.acc = [[t2.path[0][1]], t2.path[1][:2]], [1, 2]
    t2.tail_counts.fill_(0)
    t2.check(mo, torch.full_like(t2.tail_mass, -7.0), 0.0)
    # keys with infinities: weight 0 where the logit is -inf, NaN where it is NaN
    t3 = Masses(9, "bf16", 1, 2, 1, 128, [[[40]]], [1], [5])
    t3.Q[..., 0] = 1.0
    t3.Kc[3, 0], t3.Kc[4, 0] = -float("inf"), float("nan")
    mo, _ = t3.run(1.0)
    assert float(mo[3]) == float(t3.mass[3]) and bool(mo[4].isnan()) and int(mo.isnan().sum()) == 1


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_accumulate_queries_that_weigh_nothing(dtype, D):
    """Whatever a query holds that a path leaves out, that saw no row or that only fills a tile."""
    say(f"accumulate, queries that weigh nothing {dtype} {D}")
    t = Masses(11, dtype, 1, 4, 2, D, [[[90], [80]]], [3], [40, 41, 9], 5, page=8, accepted=[2, 3, 0])
    want = t.run(0.5)
    t.check(*want, 0.5)
    t.path_t[0, 2], t.path_t[1, 3], t.path_t[2, 0] = 5, -1, 99           # not accepted: not read
    t.acc_t[0], t.acc_t[1] = 3, 4
    for c, k in ((0, 2), (1, 3)):                                      # accepted, not there
        t.path[c], t.acc[c] = t.path[c][:k], k
    used = {c * 5 + v for c in range(3) for v in t.path[c][:t.acc[c]]}
    for q in set(range(15)) - used:
        t.Q[:, :, q], t.lse[:, :, q] = float("nan"), float("inf")
    got = t.run(0.5)
    t.check(*got, 0.5, skip_conts=(0, 1))                                # (the sums' order is another)
    # a node that saw no row: its query does not matter either
    gone = t.path[1][1]
    t.lse[:, :, 5 + gone] = -float("inf")
    clean = t.run(0.5)[0]
    t.Q[:, :, 5 + gone] = float("nan")
    got = t.run(0.5)[0]
    assert torch.equal(got, clean) and not torch.equal(got, want[0]) and bool(got[:170].isfinite().all())
    # and where rows hold infinities, so that products with nothing are NaN
    t.Kc[5, 3] = float("inf")
    got = t.run(0.5)[0]
    assert not bool(got.isnan().any()) and torch.equal(torch.cat([got[:5], got[6:170]]), torch.cat([clean[:5], clean[6:170]]))


def test_accumulate_without_continuations():
    """Prompts that nobody continues only fade."""
    say("accumulate, no continuations")
    t = Masses(10, "bf16", 1, 4, 2, 64, [[[90, 50], [80, 40]]], [0, 2], [3, 4])
    mo, to = t.run(0.25)
    t.check(mo, to, 0.25)
    assert torch.equal(mo[:90], 0.25 * t.mass[:90])


# ---------------------------------------------------------------------------

def expected(mass, n, limit, keep, recent):
    """Where each row of a unit afterwards comes from, or None: as it was."""
    if n <= limit:
        return None
    heavy, old = keep - recent, n - recent
    key = lambda r: (-float("inf") if mass[r] != mass[r] else mass[r] + 0.0)  # noqa: E731
    # (NaN below -inf: a second key)
    order = sorted(range(old), key=lambda r: (mass[r] != mass[r], -key(r), r))
    stays = set(order[:heavy])
    src = list(range(heavy)) + list(range(old, n))
    free = [r for r in range(heavy) if r not in stays]
    late = sorted(r for r in stays if r >= heavy)
    assert len(free) == len(late)
    for a, b in zip(free, late):
        src[a] = b
    return src


def masses(kind, g, shape):
    m = torch.randn(shape, generator=g, device="cuda").exp()
    if kind == "ties":
        m = (m * 2).round() / 2
    elif kind == "odd":
        u = torch.rand(shape, generator=g, device="cuda")
        for lo, v in ((0.1, float("nan")), (0.2, 0.0), (0.3, -0.0), (0.35, float("inf")), (0.4, -float("inf")), (0.45, -1.0), (0.5, 1e-42)):
            m = torch.where((u < lo) & (u >= lo - 0.1), v, m)
    elif kind == "same":
        m = torch.ones_like(m)
    elif kind == "old":  # the lightest first: the most rows move
        m = m.flatten().sort().values.view(shape)
    return m


def check_unit(K, V, m, K2, V2, m2, n, limit, keep, recent, bits, same_buffer):
    """Rows of one unit before and after."""
    src = expected(m.tolist(), n, limit, keep, recent)
    if src is None:
        assert torch.equal(K.view(bits), K2.view(bits)) and torch.equal(V.view(bits), V2.view(bits))
        assert torch.equal(m[:n].view(torch.int32), m2[:n].view(torch.int32))
        return n
    for x, y in ((K, K2), (V, V2)):
        assert torch.equal(x[src].view(bits), y[:keep].view(bits))
    assert torch.equal(m[src].view(torch.int32), m2[:keep].view(torch.int32))
    if not same_buffer:
        assert bool((m2[keep:] == -7).all())
    return keep


TAILS = [  # dtype, L, Hkv, D, page, limit, keep, recent, tails, masses
    ("bf16", 2, 4, 128, 64, 1024, 1024, 128, [1152, 1151, 1024, 1000, 1025, 5], "plain"),
    ("bf16", 1, 2, 64, 1, 40, 30, 25, [41, 50, 300, 40, 0, 1], "ties"),
    ("f32", 3, 2, 128, 16, 256, 200, 0, [300, 257, 256], "plain"),
    ("f32", 1, 1, 64, 8, 64, 64, 64, [65, 100, 2000], "odd"),
    ("bf16", 1, 2, 128, 32, 100, 100, 1, [3000, 1025, 101], "same"),
    ("bf16", 1, 3, 64, 4, 1, 1, 0, [2, 900, 1], "odd"),
    ("bf16", 1, 2, 64, 16, 1, 1, 1, [2, 900, 1], "plain"),
    ("bf16", 1, 1, 128, 256, 9000, 9000, 77, [20000, 9001], "ties"),
    ("f32", 1, 2, 128, 16, 2500, 2500, 2000, [2600, 4999, 2501], "old"),
    ("bf16", 2, 1, 64, 64, 700, 350, 349, [701, 1400], "old"),
    # many units
    ("bf16", 28, 4, 64, 16, 200, 150, 40, [201, 300, 150, 90, 777], "ties"),
    ("f32", 32, 4, 128, 8, 300, 300, 290, [310, 301, 1, 590], "odd"),
    ("bf16", 16, 32, 64, 64, 20, 10, 0, [21, 2048], "same"),
]


@pytest.mark.parametrize("case", TAILS, ids=lambda c: f"{c[0]}-L{c[1]}-h{c[2]}-D{c[3]}-p{c[4]}-{c[5]}-{c[6]}-{c[7]}-{c[9]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_tails(case, in_place):
    import paper_2609_06663_amd as P
    dtype, L, Hkv, D, page, limit, keep, recent, tails, kind = case
    say(f"tails {case} {in_place}")
    t = Cache(5, dtype, L, Hkv, Hkv, D, [[[1]] * Hkv] * L, [len(tails)], tails, page=page)
    mass = masses(kind, t.g, t.tk.shape[:-1])
    K, V, m = t.tk.clone(), t.tv.clone(), mass.clone()
    out = mass if in_place else torch.full_like(mass, -7.0)
    counts = t.tail_counts.clone()
    new = counts if in_place else torch.full_like(counts, -7)
    ws = torch.full((max(256, P.ecokv_evict_workspace_size(t.shape, t.N, t.max_tail, keep)),), 0xFF, dtype=torch.uint8, device="cuda")
    P.ecokv_evict_tails(t.shape, t.tails, counts, t.max_tail, limit, keep, recent, mass, new, out, ws)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert new.tolist() == [keep if n > limit else n for n in tails]
    for c, n in enumerate(tails):
        p, r = t.tail_index(c, list(range(n)))
        for l in range(L):
            for h in range(Hkv):
                check_unit(K[l, p, h, r], V[l, p, h, r], m[l, p, h, r], t.tk[l, p, h, r], t.tv[l, p, h, r], out[l, p, h, r], n, limit, keep,
                           recent, bits, in_place)
    # rows of nobody are left as they were
    other = torch.ones(t.tk.shape[1], page, dtype=torch.bool, device="cuda")
    for c, n in enumerate(tails):
        p, r = t.tail_index(c, list(range(n)))
        other[p, r] = False
    for x, y in ((K, t.tk), (V, t.tv)):
        assert torch.equal(x.permute(1, 3, 0, 2, 4)[other].view(bits), y.permute(1, 3, 0, 2, 4)[other].view(bits))


KEPT = [  # dtype, L, Hkv, D, limit, keep, recent, counts (per prompt), masses
    ("bf16", 2, 4, 128, 500, 400, 8, [900, 500, 501, 0, 1], "plain"),
    ("f32", 1, 2, 64, 2000, 2000, 0, [6553, 2001], "ties"),
    ("bf16", 1, 1, 128, 17, 16, 16, [6000, 18], "odd"),
    ("bf16", 4, 8, 128, 2047, 2047, 8, [2800, 4000], "old"),
    ("bf16", 32, 8, 64, 100, 80, 70, [300, 120, 90], "ties"),
    ("f32", 32, 8, 64, 1000, 1000, 1, [1300, 1001], "odd"),
]


@pytest.mark.parametrize("case", KEPT, ids=lambda c: f"{c[0]}-L{c[1]}-h{c[2]}-D{c[3]}-{c[4]}-{c[5]}-{c[6]}-{c[8]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_kept(case, in_place):
    import paper_2609_06663_amd as P
    dtype, L, Hkv, D, limit, keep, recent, counts, kind = case
    say(f"kept {case} {in_place}")
    t = Cache(6, dtype, L, Hkv, Hkv, D, ragged(counts, L, Hkv), [1] * len(counts), [1] * len(counts))
    mass = masses(kind, t.g, (t.Kc.shape[0],))
    K, V, m = t.Kc.clone(), t.Vc.clone(), mass.clone()
    out = mass if in_place else torch.full_like(mass, -7.0)
    before = t.counts.tolist()
    new = t.counts if in_place else torch.full_like(t.counts, -7)
    P.ecokv_evict(t.Kc, t.Vc, t.shape, t.counts, t.offsets, t.max_count, limit, keep, recent, mass, new, out)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert new.tolist() == [keep if n > limit else n for n in before]
    for n, o in zip(before, t.offsets.tolist()):
        s = slice(o, o + n)
        check_unit(K[s], V[s], m[s], t.Kc[s], t.Vc[s], out[s], n, limit, keep, recent, bits, in_place)


def test_evict_leaves_alone_what_it_should():
    """Counts out of their bounds, tails with a page that is not there."""
    import paper_2609_06663_amd as P
    say("evict, out of bounds")
    t = Cache(7, "bf16", 2, 2, 2, 64, [[[90, 50, 30], [80, 40, 20]], [[90, 50, 30], [80, 40, 20]]], [1, 1, 1], [60, 61, 90], page=8)
    K, V = t.Kc.clone(), t.Vc.clone()
    mass = masses("plain", t.g, (t.Kc.shape[0],))
    m = mass.clone()
    t.counts[0], t.counts[4] = t.max_count + 1, -5
    P.ecokv_evict(t.Kc, t.Vc, t.shape, t.counts, t.offsets, t.max_count, 1000, 35, 5, mass)
    assert torch.equal(K, t.Kc) and torch.equal(V, t.Vc) and torch.equal(m, mass)  # (none is past the limit)
    new = torch.empty_like(t.counts)
    P.ecokv_evict(t.Kc, t.Vc, t.shape, t.counts, t.offsets, t.max_count, 35, 35, 5, mass, new)
    assert new.tolist() == [91, 35, 30, 35, -5, 20, 35, 35, 30, 35, 35, 20]
    for u in (0, 4):
        s = slice(int(t.offsets[u]), int(t.offsets[u]) + [90, 0, 0, 0, 40][u])
        assert torch.equal(K[s], t.Kc[s]) and torch.equal(V[s], t.Vc[s]) and torch.equal(m[s], mass[s])
    tm = masses("plain", t.g, t.tk.shape[:-1])
    t.table[1, 7] = -1           # row 60, the last of continuation 1
    t.tail_counts[2] = 91        # past the bound
    K, V, m = t.tk.clone(), t.tv.clone(), tm.clone()
    P.ecokv_evict_tails(t.shape, t.tails, t.tail_counts, 90, 20, 20, 3, tm)
    assert t.tail_counts.tolist() == [20, 61, 91]
    for c in (1, 2):
        p = t.table[c].long().clamp_min(0)
        p = p[t.table[c] >= 0]
        assert torch.equal(K[:, p].view(torch.int16), t.tk[:, p].view(torch.int16)) and torch.equal(m[:, p], tm[:, p])
    assert not torch.equal(K.view(torch.int16), t.tk.view(torch.int16))
