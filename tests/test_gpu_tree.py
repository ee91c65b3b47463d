"""ecokv_decode_tree against attention in 64 bits, and ecokv_commit against moved
rows, at the sizes, trees, splits, pages and values where they can go wrong.

Tolerance.  dx bounds a logit's error (cache_cases.logit_error).  A weight's relative
error is at most 2 dx beside its normalisation, weighted sums and merges add fewer
than 64 roundings; with bf16 rows a weight w_j is rounded to bf16 in its product with
the values, half a step of 2^-8 w_j, and O once more at the end:
  |O - O64| <= (2 dx + 2^-18) max |V| [+ 2^-8 (1 + 2^-6) (sum_j w_j |v_j| + |O64|)],
  |lse - lse64| <= dx + 2^-20 max(1, |lse64|).
"""
import random
import sys

import pytest
import torch

from cache_cases import Cache, logit_error, random_tree, signed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-tree] {msg}", file=sys.stderr, flush=True)


def masks_of(kind, N, M, seed):
    """[N][M] Python integers: trees, any bits at all, or nothing."""
    import paper_2609_06663_amd as P
    rng = random.Random(seed)
    out = []
    for c in range(N):
        if kind == "tree":
            live = M if c % 3 else rng.randint(1, M)
            m = [v & (2 ** 64 - 1) for v in P.ecokv_tree_masks(random_tree(rng, live))[0]] + [0] * (M - live)
        elif kind == "any":
            m = [rng.getrandbits(64) if rng.random() < 0.8 else 0 for _ in range(M)]
        else:
            m = [0] * M
        out.append(m)
    return out


class Trees(Cache):
    def __init__(self, seed, dtype, L, Hq, Hkv, D, counts, fan, tails, nodes, kind="tree", **kw):
        super().__init__(seed, dtype, L, Hq, Hkv, D, counts, fan, tails, nodes, **kw)
        self.bits = masks_of(kind, self.N, nodes, seed)
        self.masks = torch.tensor([[signed(m) for m in row] for row in self.bits], dtype=torch.int64).view(self.N, nodes).cuda()
        self.Q = torch.randn((L, Hq, self.N * nodes, D), generator=self.g, device="cuda").to(self.type)
        # drafted rows that no node sees may hold anything
        for c in range(self.N):
            seen = 0
            for m in self.bits[c]:
                seen |= m
            hidden = [tails[c] + j for j in range(nodes) if not (seen >> j) & 1]
            if hidden and tails[c] >= 0:
                p, r = self.tail_index(c, hidden)
                self.tk.permute(1, 3, 0, 2, 4)[p, r] = float("nan")
                self.tv.permute(1, 3, 0, 2, 4)[p, r] = float("inf")

    def run(self, stream=None, out=None, **kw):
        import paper_2609_06663_amd as P
        L, Hq, _, D, _ = self.dims
        O, lse = out or (torch.full((L, Hq, self.N * self.nodes, D), -7.0, device="cuda", dtype=self.type),
                         torch.full((L, Hq, self.N * self.nodes), -7.0, device="cuda"))
        mc, mt = kw.get("max_count", self.max_count), kw.get("max_tail", self.max_tail)
        ws = torch.full((max(256, P.ecokv_decode_tree_workspace_size(self.shape, self.fan, mc, mt, self.nodes)),), 0xFF, dtype=torch.uint8, device="cuda")
        P.ecokv_decode_tree(self.Q, self.Kc, self.Vc, self.shape, self.fan, self.counts, self.offsets, mc, self.tails, self.tail_counts, mt,
                            self.masks, O, lse, ws, stream)
        torch.cuda.synchronize()
        return O, lse

    def reference(self, l, h, c):
        """Logits [M][G][rows] in 64 bits, -inf where hidden, the rows' K and V, and what was seen [M][rows]."""
        L, Hq, Hkv, D, _ = self.dims
        G, M, n = Hq // Hkv, self.nodes, int(self.tail_counts[c])
        a = self.kept(l, h, c)
        p, r = self.tail_index(c, list(range(n + M)))
        K, V = (torch.cat([x[a], y[l, p, h, r]]).double() for x, y in ((self.Kc, self.tk), (self.Vc, self.tv)))
        seen = torch.ones((M, len(K)), dtype=torch.bool)
        seen[:, len(K) - M:] = torch.tensor([[(m >> j) & 1 == 1 for j in range(M)] for m in self.bits[c]])
        seen = seen.cuda()
        q = self.Q[l, h * G:(h + 1) * G, c * M:(c + 1) * M].double().transpose(0, 1)
        x = (q.reshape(M * G, D) @ K.t() / D ** 0.5).view(M, G, -1)
        return x.masked_fill(~seen[:, None], -float("inf")), K, V, seen, q

    def check(self, O, lse, skip=()):
        L, Hq, Hkv, D, _ = self.dims
        G, M, bf = Hq // Hkv, self.nodes, self.type == torch.bfloat16
        for l in range(L):
            for h in range(Hkv):
                for c in range(self.N):
                    if c in skip:
                        continue
                    x, K, V, seen, q = self.reference(l, h, c)
                    got = O[l, h * G:(h + 1) * G, c * M:(c + 1) * M].double().transpose(0, 1)
                    gl = lse[l, h * G:(h + 1) * G, c * M:(c + 1) * M].double().t()
                    none = ~seen.any(1)
                    assert bool((got[none] == 0).all()) and bool((gl[none] == -float("inf")).all()), (l, h, c)
                    live = ~none
                    if not bool(live.any()):
                        continue
                    rows = seen.any(0)
                    K, V = torch.where(rows[:, None], K, 0.0), torch.where(rows[:, None], V, 0.0)
                    w = x[live].softmax(-1)
                    ref, rl = w @ V, x[live].logsumexp(-1)
                    dx = logit_error(q.reshape(M * G, D), K, D)
                    tol = (2 * dx + 2.0 ** -18) * float(V.abs().max()) + (2.0 ** -8 * (1 + 2.0 ** -6) * (w @ V.abs() + ref.abs()) if bf else 0)
                    err = (got[live] - ref).abs()
                    assert bool((err <= tol).all()), (l, h, c, float((err - tol).max()), dx)
                    assert bool(((gl[live] - rl).abs() <= dx + 2.0 ** -20 * rl.abs().clamp_min(1)).all()), (l, h, c)


SHAPES = [  # dtype, D, L, Hq, Hkv, counts (per unit), fan, tails, nodes, page
    ("bf16", 128, 1, 28, 4, [6553], [1], [700], 64, 64),
    ("bf16", 128, 1, 28, 4, [700, 33], [3, 2], [5, 16, 17, 0, 129], 7, 16),
    ("bf16", 128, 2, 32, 8, [1500, 1, 64, 0, 129], [2, 1, 3, 0, 3], [7 * i % 50 for i in range(9)], 13, 8),
    ("bf16", 64, 1, 8, 8, [2049], [5], [100, 63, 64, 65, 1], 33, 1),
    ("bf16", 64, 3, 6, 2, [40, 257], [1, 1], [300, 2], 2, 128),
    ("bf16", 128, 1, 64, 1, [1000], [2], [40, 33], 31, 16),
    ("bf16", 128, 1, 17, 1, [515], [9], [3 * i for i in range(9)], 1, 4),
    ("bf16", 128, 1, 4, 2, [2000], [6], [311 * i for i in range(6)], 16, 32),
    ("bf16", 128, 1, 1, 1, [31], [1], [1], 1, 16),
    ("f32", 128, 1, 8, 4, [300, 20], [3, 2], [50, 0, 1, 17, 16], 5, 16),
    ("f32", 128, 1, 2, 2, [128], [2], [5, 4], 64, 16),
    ("f32", 64, 2, 12, 4, [1, 515], [4, 1], [30 * i for i in range(5)], 9, 2),
    ("f32", 64, 1, 40, 1, [900], [2], [200, 1], 12, 64),
    ("f32", 128, 1, 28, 4, [211], [3], [9, 70, 150], 3, 16),
]
IDS = dict(ids=lambda c: f"{c[0]}-D{c[1]}-L{c[2]}-{c[3]}q{c[4]}kv-{c[5]}-{c[6]}-m{c[8]}-p{c[9]}")


def ragged(counts, L, Hkv):
    return [[[max(0, n - 13 * ((3 * h + l) % 4)) if n > 60 else n for n in counts] for h in range(Hkv)] for l in range(L)]


@pytest.mark.parametrize("case", SHAPES, **IDS)
@pytest.mark.parametrize("kind", ["tree", "any"])
def test_tree(case, kind):
    dtype, D, L, Hq, Hkv, counts, fan, tails, nodes, page = case
    say(f"{case[:9]} page {page} {kind}")
    t = Trees(7, dtype, L, Hq, Hkv, D, ragged(counts, L, Hkv), fan, tails, nodes, kind, page=page, kscale=1.0 if kind == "tree" else 6.0)
    O, lse = t.run()
    t.check(O, lse)
    # bounds above the counts split the rows otherwise
    O2, lse2 = t.run(max_count=4 * t.max_count + 900, max_tail=t.table.shape[1] * page)
    t.check(O2, lse2)
    # and a second call gives the same bits
    O3, lse3 = t.run()
    assert torch.equal(O, O3) and torch.equal(lse, lse3)


@pytest.mark.parametrize("case", SHAPES, **IDS)
def test_tree_as_in_large_calls(case):
    # a bound of 3 million kept rows: split like a call that reads gigabytes
    dtype, D, L, Hq, Hkv, counts, fan, tails, nodes, page = case
    say(f"{case[:9]} page {page}, split for 3 million rows")
    t = Trees(20, dtype, L, Hq, Hkv, D, [[counts] * Hkv] * L, fan, tails, nodes, page=page)
    t.check(*t.run(max_count=3_000_000))


@pytest.mark.parametrize("dtype,D,L,Hq,Hkv,nodes,fan", [
    ("bf16", 128, 1, 32, 8, 13, [5, 1, 6, 2, 0]),
    ("bf16", 64, 3, 8, 4, 30, [1, 0, 2, 1, 1]),
    ("bf16", 128, 1, 28, 4, 3, [9, 30, 4, 1, 2]),
    ("f32", 128, 1, 16, 4, 7, [4, 2, 1, 3, 1]),
    ("f32", 64, 2, 6, 2, 20, [1, 1, 2, 0, 1]),
])
def test_prompts_of_different_lengths(dtype, D, L, Hq, Hkv, nodes, fan):
    """Long and short units, units without rows, bounds far above the counts."""
    say(f"different lengths {dtype} {D} {L} {Hq}/{Hkv} {nodes} {fan}")
    counts = [[[4480 - 97 * (h + l), 3 * h, 619 + h, max(0, 2610 - 900 * h), 1] for h in range(Hkv)] for l in range(L)]
    t = Trees(23, dtype, L, Hq, Hkv, D, counts, fan, [7 * c % 50 for c in range(sum(fan))], nodes, page=16)
    for bound in (4480, 20_000, 300_000):
        O, lse = t.run(max_count=bound)
        t.check(O, lse)
        again = t.run(max_count=bound)
        assert torch.equal(O, again[0]) and torch.equal(lse, again[1])
    # lengths change between calls: nothing of the last one's split stays
    c = t.counts.clone()
    t.counts.copy_(torch.where(torch.arange(len(c), device="cuda") % 3 == 0, c // 5, c))
    t.check(*t.run(max_count=20_000))
    t.counts.zero_()
    t.check(*t.run(max_count=20_000))
    t.counts.copy_(c)
    t.counts[0], t.counts[7] = 20_001, -1     # head 0's prompt 0, head 1's prompt 2
    O, lse = t.run(max_count=20_000)
    G, bad = Hq // Hkv, []
    for h, s in ((0, 0), (1, 2)):
        for k in range(t.fan[s], t.fan[s + 1]):
            at = (0, slice(h * G, (h + 1) * G), slice(k * nodes, (k + 1) * nodes))
            assert bool(O[at].isnan().all()) and bool(lse[at].isnan().all())
            bad.append(k)
    t.check(O, lse, skip=bad)


@pytest.mark.parametrize("dtype,D,nodes", [("bf16", 128, 24), ("bf16", 64, 40), ("bf16", 128, 3), ("f32", 128, 24), ("f32", 64, 24)])
def test_any_number_of_parts(dtype, D, nodes):
    """Bounds from the counts up to many times them: one part of a tail to more than 32, few of them with rows."""
    import paper_2609_06663_amd as P
    t = Trees(21, dtype, 1, 8, 2, D, [[[40], [300]]], [2], [40, 3], nodes, page=16, spare=9000)
    seen = set()
    for most in (40, 100, 150, 200, 300, 400, 600, 900, 1200, 1700, 2500, 4000, 9000):
        say(f"{dtype} {D} {nodes}: tails of up to {most} rows")
        t.check(*t.run(max_tail=most))
        seen.add(P.ecokv_decode_tree_workspace_size(t.shape, t.fan, t.max_count, most, nodes) // (8 * 2 * nodes * 4 * (D + 2)))
    assert min(seen) <= 5 and max(seen) > 32 and len(seen) > 6


@pytest.mark.parametrize("dtype,D,Hq,Hkv,nodes", [("bf16", 128, 28, 4, 9), ("bf16", 64, 4, 4, 64), ("f32", 128, 6, 2, 3), ("f32", 64, 8, 1, 20)])
def test_tails_alone(dtype, D, Hq, Hkv, nodes):
    say(f"tails alone {dtype} {D} {nodes}")
    t = Trees(3, dtype, 2, Hq, Hkv, D, [[[0]] * Hkv] * 2, [5], [0, 1, 40, 1000, 2111], nodes, "any", page=32)
    assert t.max_count == 0
    t.Kc = t.Vc = t.counts = t.offsets = None  # (not read)
    t.kept = lambda l, h, c: slice(0, 0)
    t.Kc = t.Vc = torch.zeros((0, D), dtype=t.type, device="cuda")
    t.check(*t.run())


@pytest.mark.parametrize("dtype,G,nodes", [("bf16", 1, 1), ("bf16", 7, 64), ("f32", 4, 2), ("f32", 1, 40)])
def test_nothing_to_see(dtype, G, nodes):
    say(f"no rows {dtype} {G} {nodes}")
    t = Trees(4, dtype, 1, 2 * G, 2, 64, [[[0], [0]]], [3], [0, 0, 0], nodes, "none")
    O, lse = t.run()
    assert bool((O == 0).all()) and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("dtype,D,G,nodes", [("bf16", 128, 1, 8), ("bf16", 128, 7, 40), ("bf16", 64, 2, 64), ("f32", 64, 1, 8), ("f32", 128, 8, 33)])
def test_values_that_are_not_finite(dtype, D, G, nodes):
    """Drafted rows with infinities and NaN reach the nodes that see them, in those dimensions alone, and nobody else."""
    say(f"not finite {dtype} {D} {G} {nodes}")
    t = Trees(11, dtype, 1, 2 * G, 2, D, [[[70], [33]]], [2], [45, 3], nodes, "any", page=8)
    odd = [(0, 1, 5, float("inf")), (0, nodes - 1, 6, float("nan")), (1, 0, D - 1, -float("inf")), (1, 3, 0, float("inf")), (1, 4, 0, -float("inf"))]
    for c, j, d, v in odd:
        p, r = t.tail_index(c, [int(t.tail_counts[c]) + j])
        t.tv[:, p, :, r, d] = v
    O, lse = t.run()
    assert not bool(lse.isnan().any())
    clean = O.clone()
    for c in range(2):
        for i in range(nodes):
            want = {}
            for cc, j, d, v in odd:
                if cc == c and (t.bits[c][i] >> j) & 1:
                    want[d] = v if d not in want else float("nan")
            got = O[0, :, c * nodes + i].float()
            for d, v in want.items():
                assert bool((got[:, d].isnan() if v != v else got[:, d] == v).all()), (c, i, d, v, got[:, d])
                clean[0, :, c * nodes + i, d] = 0
    assert bool(clean.isfinite().all())
    # the others are what they would be without
    for c, j, d, v in odd:
        p, r = t.tail_index(c, [int(t.tail_counts[c]) + j])
        t.tv[:, p, :, r, d] = 0
    O2, lse2 = t.run()
    t.check(O2, lse2)
    keep = O.isfinite()
    assert torch.equal(O[keep], O2[keep]) and torch.equal(lse, lse2)
    # a key that is not finite: the nodes that see it alone
    p, r = t.tail_index(0, [int(t.tail_counts[0]) + 2])
    t.tk[:, p, :, r, 1] = float("nan")
    O3, lse3 = t.run()
    sees = torch.tensor([(t.bits[0][i] >> 2) & 1 == 1 for i in range(nodes)] + [False] * nodes, device="cuda")
    assert bool(O3[0][:, sees].isnan().all()) and bool(lse3[0][:, sees].isnan().all())
    assert torch.equal(O3[0][:, ~sees], O2[0][:, ~sees]) and torch.equal(lse3[0][:, ~sees], lse2[0][:, ~sees])


@pytest.mark.parametrize("dtype,G,nodes", [("bf16", 1, 6), ("bf16", 7, 64), ("f32", 2, 40)])
def test_counts_and_pages_out_of_bounds(dtype, G, nodes):
    say(f"out of bounds {dtype} {G} {nodes}")
    t = Trees(12, dtype, 1, 2 * G, 2, 128, [[[90, 50, 30], [80, 40, 20]]], [2, 2, 2], [40, 41, 90, 43, 17, 30], nodes, "any", page=8)
    t.counts[1] = t.max_count + 1                # prompt 1, head 0: continuations 2 and 3
    t.tail_counts[0] = -1                        # continuation 0
    t.table[4, 1] = t.tk.shape[1]                # a tail page of continuation 4
    t.table[5, (30 + 2) // 8] = -1               # a page of drafted rows 2 .. 9 of continuation 5 (rows 32 .. 39)
    O, lse = t.run()
    M = nodes
    nan = lambda x: bool(x.isnan().all())  # noqa: E731
    assert nan(O[0, :, :M]) and nan(lse[0, :, :M])
    assert nan(O[0, :G, 2 * M:4 * M]) and nan(lse[0, :G, 2 * M:4 * M])
    assert nan(O[0, :, 4 * M:5 * M]) and nan(lse[0, :, 4 * M:5 * M])
    lost = [any((t.bits[5][i] >> j) & 1 for j in range(2, min(10, M))) for i in range(M)]
    lost = torch.tensor(lost, device="cuda")
    assert nan(O[0][:, 5 * M:][:, lost]) and nan(lse[0][:, 5 * M:][:, lost])
    assert bool(O[0][:, 5 * M:][:, ~lost].isfinite().all())
    t.check(O, lse, skip=(0, 2, 3, 4, 5))
    O2, _ = t.run(max_tail=60)  # continuation 2 has 90 rows
    assert nan(O2[0, G:, 2 * M:3 * M])


def test_one_node_is_decode_shared():
    """A node that sees itself: the same attention as of one generated token."""
    import paper_2609_06663_amd as P
    say("one node")
    t = Trees(13, "f32", 2, 8, 2, 128, [[[300], [200]], [[100], [301]]], [4], [10, 0, 33, 64], 1, page=16)
    t.masks.fill_(1)
    O, lse = t.run()
    O2, lse2 = torch.empty_like(O), torch.empty_like(lse)
    P.ecokv_decode_shared(t.Q, t.Kc, t.Vc, t.shape, t.fan, t.counts, t.offsets, t.max_count, t.tails, t.tail_counts + 1, t.max_tail + 1, O2, lse2)
    # (both are within 2 dx + 2^-18 of the exact values; dx < 2^-16 for these)
    assert float((O - O2).abs().max()) <= 4 * (2.0 ** -15 + 2.0 ** -18) * 5 and float((lse - lse2).abs().max()) <= 2.0 ** -14


def test_forks_share_pages():
    """Two continuations whose tails begin with the same pages."""
    say("forks")
    t = Trees(14, "bf16", 1, 8, 2, 128, [[[64], [64]]], [2], [32, 40], 6, page=16)
    t.table[1, :2] = t.table[0, :2]
    t.check(*t.run())


def test_past_32_bits():
    """A pool whose last pages lie past 2^32 bytes, in both K and V."""
    say("a pool past 32 bits")
    import paper_2609_06663_amd as P
    t = Trees(15, "bf16", 1, 8, 8, 128, [[[5]] * 8], [2], [100, 37], 20, page=64)
    pages = (2 ** 32 + 2 ** 26) // (8 * 64 * 128 * 2)
    used = t.tk.shape[1]
    K, V = (torch.zeros((1, pages, 8, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[:, pages - used:], V[:, pages - used:] = t.tk, t.tv
    t.tk, t.tv, t.table = K, V, t.table + (pages - used)
    t.tails = P.Tails(K, V, t.table)
    t.check(*t.run())


# ---------------------------------------------------------------------------

def commit_case(seed, dtype, L, Hkv, D, tails, nodes, page):
    t = Cache(seed, dtype, L, Hkv, Hkv, D, [[[1]] * Hkv] * L, [len(tails)], tails, nodes, page=page)
    rng = random.Random(seed)
    path, acc = [], []
    for c in range(t.N):
        a = [0, nodes, 1, rng.randint(0, nodes)][c % 4]
        p = sorted(rng.sample(range(nodes), a))
        if c % 5 == 3:
            p = list(range(a))  # (nothing moves)
        path.append(p + [nodes + 7] * (nodes - a))
        acc.append(a)
    t.path, t.acc = path, acc
    return t


def run_commit(t, path=None, accepted=None):
    import paper_2609_06663_amd as P
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    P.ecokv_commit(t.shape, t.tails, t.tail_counts, i32(path or t.path).view(t.N, -1), i32(accepted or t.acc))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,L,Hkv,D,nodes,page", [("bf16", 3, 4, 128, 64, 16), ("bf16", 1, 2, 64, 7, 1), ("f32", 2, 3, 128, 64, 8), ("f32", 1, 1, 64, 1, 32),
                                                      ("bf16", 28, 4, 128, 5, 64)])
def test_commit(dtype, L, Hkv, D, nodes, page):
    say(f"commit {dtype} {L} {Hkv} {D} {nodes} {page}")
    t = commit_case(9, dtype, L, Hkv, D, [0, 1, 30, 17, 64, 5, 99, 16, 15], nodes, page)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    want = [x.clone() for x in (t.tk, t.tv)]
    for c in range(t.N):
        n = int(t.tail_counts[c])
        p, r = t.tail_index(c, [n + v for v in t.path[c][:t.acc[c]]])
        q, s = t.tail_index(c, [n + k for k in range(t.acc[c])])
        for x, y in zip((t.tk, t.tv), want):
            y.permute(1, 3, 0, 2, 4)[q, s] = x.permute(1, 3, 0, 2, 4)[p, r]
    run_commit(t)
    for x, y in zip((t.tk, t.tv), want):
        assert torch.equal(x.view(bits), y.view(bits))


def test_commit_leaves_alone_what_it_should():
    say("commit, bad paths and pages")
    t = commit_case(10, "bf16", 2, 2, 64, [20, 21, 22, 23, 24, 25, 26, 27], 8, 8)
    path = [[1, 3, 5, 0, 0, 0, 0, 0],      # good
            [1, 3, 3, 0, 0, 0, 0, 0],      # twice the same
            [3, 1, 5, 0, 0, 0, 0, 0],      # not ascending
            [1, 3, 8, 0, 0, 0, 0, 0],      # past the nodes
            [-1, 3, 5, 0, 0, 0, 0, 0],     # below
            [1, 3, 5, 0, 0, 0, 0, 0],      # accepted out of range (9)
            [1, 3, 5, 0, 0, 0, 0, 0],      # a page that is not there
            [1, 3, 5, 0, 0, 0, 0, 0]]      # a negative count
    acc = [3, 3, 3, 3, 3, 9, 3, 3]
    t.table[6, 3] = t.tk.shape[1]  # rows 24 .. 31
    t.tail_counts[7] = -3
    want = [x.clone() for x in (t.tk, t.tv)]
    p, r = t.tail_index(0, [21, 23, 25])
    q, s = t.tail_index(0, [20, 21, 22])
    for x, y in zip((t.tk, t.tv), want):
        y.permute(1, 3, 0, 2, 4)[q, s] = x.permute(1, 3, 0, 2, 4)[p, r]
    run_commit(t, path, acc)
    for x, y in zip((t.tk, t.tv), want):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
