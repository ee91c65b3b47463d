"""Generation with drafted trees and a cache that stays bounded, as a program does
it: prefill -> score, select, compact -> drafts, commits, accumulated weights and
evictions between ordinary steps (pipeline.Continuations), each call checked against
64 bits with the tolerances of its own tests; captured in HIP graphs and replayed;
on other streams and several at once; in pools past 32 bits."""
import random
import sys

import pytest
import torch

from cache_cases import Cache, random_tree
from test_gpu_evict import Masses, check_unit
from test_gpu_generate import Model, check_step
from test_gpu_rope import near, turned
from test_gpu_tree import Trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-drafts] {msg}", file=sys.stderr, flush=True)


def as_case(cls, co, **kw):
    """The state of Continuations as a case of the operators' own tests."""
    c, v = co.ep.shape.c, cls.__new__(cls)
    v.dims = (c.num_layers, c.num_q_heads, c.num_kv_heads, c.head_dim, c.num_seqs)
    v.fan, v.N, v.type, v.page = co.fan, co.fan[-1], co.Q_dec.dtype, co.tails.K.shape[3]
    v.Kc, v.Vc, v.counts, v.offsets = co.ep.Kc, co.ep.Vc, co.ep.counts, co.ep.offsets
    v.tk, v.tv, v.table, v.tail_counts = co.tails.K, co.tails.V, co.tails.table, co.rows
    for name, x in kw.items():
        setattr(v, name, x)
    return v


class Run:
    def __init__(self, seed, dtype, L, Hq, Hkv, D, w, lens, budget, mode, fan_out, page, max_new, max_nodes):
        import paper_2609_06663_amd as P
        from paper_2609_06663_amd.pipeline import Continuations
        self.rng = random.Random(seed)
        self.m = Model(seed, dtype, L, Hq, Hkv, D, w, lens)
        self.ep = self.m.prefill(budget, {"per_head": P.PER_HEAD, "flat": P.LAYER_FLAT}[mode])
        self.fan_out, self.co = fan_out, Continuations(self.ep, fan_out, max_new, self.m.rope, page, max_nodes, True)
        self.name = "bf16" if self.m.dtype == torch.bfloat16 else "f32"

    def draft(self):
        m, co, rng = self.m, self.co, self.rng
        N, M = co.fan[-1], rng.randint(1, co.max_nodes)
        parents = [random_tree(rng, M if c == 0 else rng.randint(0, M)) for c in range(N)]
        tree = co.tree(parents)
        Q, K, V = m.project(N * M)
        before = co.rows.tolist()
        O = co.draft(Q, K, V, tree)
        bits = [[v & (2 ** 64 - 1) for v in row] for row in tree.masks.tolist()]
        t = as_case(Trees, co, Q=co.Q_nodes, nodes=M, bits=bits)
        t.check(O, co.lse_nodes)
        # what was appended, and at which positions
        rot, inter, factor, qw, kw = m.params
        depth = tree.steps[1].flatten()
        at = co.positions.repeat_interleave(M) + depth
        k, ks = turned(K, at, m.freq, rot, inter, factor, kw, 1e-6)
        q, qs = turned(Q, at, m.freq, rot, inter, factor, qw, 1e-6)
        for c in range(N):
            n = len(parents[c])
            p, r = t.tail_index(c, [before[c] + i for i in range(n)])
            i = slice(c * M, c * M + n)
            near(co.tails.K[:, p, :, r].transpose(0, 1), k[:, i], ks[:, i], self.name)
            assert torch.equal(co.tails.V[:, p, :, r].transpose(0, 1), V[:, i])
            near(co.Q_nodes[:, :, i].transpose(1, 2), q[:, i], qs[:, i], self.name)
        # a path from a root towards a leaf, for some the whole, for some nothing
        path = torch.full((N, M), 99, dtype=torch.int32)
        acc = [0] * N
        for c in range(N):
            node, chain = rng.randint(0, len(parents[c]) - 1) if parents[c] and c % 4 != 3 else -1, []
            while node >= 0:
                chain.append(node)
                node = parents[c][node]
            acc[c] = len(chain)
            path[c, :acc[c]] = torch.tensor(chain[::-1], dtype=torch.int32)
        self.path = [path[c, :acc[c]].tolist() for c in range(N)]
        want = {}
        for c in range(N):
            p, r = t.tail_index(c, [before[c] + i for i in self.path[c]])
            want[c] = co.tails.K[:, p, :, r].clone(), co.tails.V[:, p, :, r].clone()
        positions = co.positions.tolist()
        co.commit(path.cuda(), torch.tensor(acc, dtype=torch.int32, device="cuda"), longest=max(b + a for b, a in zip(before, acc)))
        assert co.rows.tolist() == [b + a for b, a in zip(before, acc)] and co.length == max(co.rows.tolist())
        assert co.positions.tolist() == [b + a for b, a in zip(positions, acc)]
        for c in range(N):
            p, r = t.tail_index(c, [before[c] + i for i in range(acc[c])])
            assert torch.equal(co.tails.K[:, p, :, r], want[c][0]) and torch.equal(co.tails.V[:, p, :, r], want[c][1])
        self.weigh(0.9, Q=co.Q_nodes, lse=co.lse_nodes, M=M, path=self.path, acc=acc)

    def step(self):
        m, co = self.m, self.co
        N = co.fan[-1]
        x = m.project(N)
        O = co.step(*x)
        # (a tree of one node that sees itself: the same rows)
        t = as_case(Trees, co, Q=co.Q_dec, nodes=1, bits=[[1]] * N)
        t.check(O, co.lse)
        if self.rng.random() < 0.5:
            co.advance()
            self.weigh(1.0, Q=co.Q_dec, lse=co.lse, M=1, path=[[0]] * N, acc=[1] * N)
        else:
            self.weigh(1.0, Q=co.Q_dec, lse=co.lse, M=1, path=[[0]] * N, acc=[1] * N, tail_counts=co.tail_counts)
            co.advance()

    def weigh(self, decay, **kw):
        co = self.co
        before = as_case(Masses, co, mass=co.mass.clone(), tail_mass=co.tail_mass.clone(), **kw)
        co.accumulate(decay)
        mass, tail_mass = co.mass, co.tail_mass
        a, b = before.check(mass, tail_mass, decay)
        assert torch.equal(mass[a], before.mass[a]) and torch.equal(tail_mass[b], before.tail_mass[b])

    def evict(self, limit, keep, recent):
        co = self.co
        t = as_case(Cache, co)
        K, V, m, rows = co.tails.K.clone(), co.tails.V.clone(), co.tail_mass.clone(), co.rows.tolist()
        at = co.positions.tolist()
        co.evict(limit, keep, recent)
        assert co.rows.tolist() == [keep if n > limit else n for n in rows] and co.positions.tolist() == at
        assert co.tail_counts.tolist() == [n + 1 for n in co.rows.tolist()] and co.length >= max(co.rows.tolist())
        bits = torch.int16 if self.name == "bf16" else torch.int32
        for l in range(t.dims[0]):
            for h in range(t.dims[2]):
                for c, n in enumerate(rows):
                    p, r = t.tail_index(c, list(range(n)))
                    check_unit(K[l, p, h, r], V[l, p, h, r], m[l, p, h, r], co.tails.K[l, p, h, r], co.tails.V[l, p, h, r],
                               co.tail_mass[l, p, h, r], n, limit, keep, recent, bits, True)
        return [n > limit for n in rows]

    def evict_kept(self, limit, keep, recent):
        co, ep = self.co, self.ep
        K, V, m, counts = ep.Kc.clone(), ep.Vc.clone(), co.mass.clone(), ep.counts.tolist()
        co.evict_kept(limit, keep, recent)
        bits = torch.int16 if self.name == "bf16" else torch.int32
        assert ep.counts.tolist() == [keep if n > limit else n for n in counts] and co.max_count >= max(ep.counts.tolist())
        for o, n in zip(ep.offsets.tolist(), counts):
            s = slice(o, o + n)
            check_unit(K[s], V[s], m[s], ep.Kc[s], ep.Vc[s], co.mass[s], n, limit, keep, recent, bits, True)


@pytest.mark.parametrize("dtype,L,Hq,Hkv,D,w,lens,budget,mode,fan_out,page,max_new,max_nodes", [
    ("bf16", 2, 28, 4, 128, 4, [1500, 700], [300, 100], "per_head", [3, 2], 4, 40, 16),
    ("bf16", 1, 8, 8, 64, 8, [900], [200], "per_head", [5], 16, 90, 64),
    ("bf16", 1, 16, 2, 128, 4, [400, 3001, 60], [80, 500, 60], "flat", [1, 0, 4], 1, 30, 9),
    ("f32", 2, 4, 2, 64, 4, [500], [100], "per_head", [2], 8, 33, 7),
])
def test_generation_that_stays_bounded(dtype, L, Hq, Hkv, D, w, lens, budget, mode, fan_out, page, max_new, max_nodes):
    say(f"{dtype} {L} layers {Hq}/{Hkv} heads of {D}: prompts {lens} -> {budget} ({mode}), continuations {fan_out}, {max_new} rows and {max_nodes} nodes")
    run = Run(1, dtype, L, Hq, Hkv, D, w, lens, budget, mode, fan_out, page, max_new, max_nodes)
    limit, keep = max_new // 2, max_new // 3
    evicted = i = 0
    while i < 14 or evicted == 0:
        assert i < 80
        if i % 3 == 2:
            run.step()
        else:
            run.draft()
        if i in (4, 9):
            most = int(run.ep.counts.max())
            run.evict_kept(most * 4 // 5, most // 2, w)
        if run.co.length > limit:
            evicted += sum(run.evict(limit, keep, keep // 4))
        i += 1
    torch.cuda.synchronize()


def test_steps_after_drafts_match_steps_alone():
    # a chain of which everything is accepted appends what as many steps do, and the
    # next step attends to the same rows
    from paper_2609_06663_amd import PER_HEAD
    from paper_2609_06663_amd.pipeline import Continuations
    m = Model(5, "f32", 2, 8, 2, 128, 4, [600, 300])
    ep = m.prefill([120, 70], PER_HEAD)
    a, b = Continuations(ep, [2, 1], 9, m.rope, 4), Continuations(ep, [2, 1], 9, m.rope, 4, 5)
    xs = [m.project(3) for _ in range(6)]
    for x in xs[:5]:
        a.step(*x)
        a.advance()
    Q, K, V = (torch.stack([x[i] for x in xs[:5]], 2).flatten(1, 2) for i in range(3))  # node i of c at 5 c + i
    b.draft(Q, K, V, b.tree([-1, 0, 1, 2, 3]))
    b.commit(torch.arange(5, dtype=torch.int32, device="cuda").expand(3, 5).contiguous(), torch.full((3,), 5, dtype=torch.int32, device="cuda"))
    a.step(*xs[5])
    b.step(*xs[5])
    torch.cuda.synchronize()
    for c in range(3):
        pa, pb = a.tails.table[c].long(), b.tails.table[c].long()
        for x, y in ((a.tails.K, b.tails.K), (a.tails.V, b.tails.V)):
            got, want = (t[:, p].transpose(1, 2).flatten(2, 3)[:, :, :6] for t, p in ((y, pb), (x, pa)))
            assert torch.equal(got, want)
    assert torch.equal(a.O, b.O) and torch.equal(a.lse, b.lse)
    check_step(m, a, [2, 1], xs[5][1], xs[5][2])
    b.length = 5
    check_step(m, b, [2, 1], xs[5][1], xs[5][2])


class Fixed:
    """Drafts of one shape, for capture: draft, then commit, weights and evictions."""

    LIMIT, KEEP, RECENT, MOST = 24, 16, 5, 40

    def __init__(self, m, ep_of, fan_out):
        from paper_2609_06663_amd.pipeline import Continuations
        self.co = Continuations(ep_of(), fan_out, self.MOST, m.rope, 4, 9, True)
        N = self.co.fan[-1]
        self.tree = self.co.tree([-1, 0, 0, 1, 2, 2, 4, 6, 3])
        self.x = [torch.zeros_like(t).contiguous() for t in m.project(9 * N)]
        self.path, self.acc = torch.zeros((N, 9), dtype=torch.int32, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")

    def put(self, x, path, acc):
        for d, s in zip((*self.x, self.path, self.acc), (*x, path, acc)):
            d.copy_(s)

    def draft(self):
        self.co.length = 0
        self.co.draft(*self.x, self.tree, max_tail=self.MOST)

    def rest(self):
        self.co.commit(self.path, self.acc)
        self.co.accumulate(0.8, max_tail=self.MOST)
        self.co.evict(self.LIMIT, self.KEEP, self.RECENT, max_tail=self.MOST)

    def state(self):
        co = self.co
        K, V, m = (torch.where(self.used()[None, :, None, :].unsqueeze(-1) if t.dim() == 5 else self.used()[None, :, None, :], t, 0)
                   for t in (co.tails.K, co.tails.V, co.tail_mass))
        return [t.clone() for t in (co.O_nodes, co.lse_nodes, co.rows, co.positions, K, V, co.mass, m)]

    def used(self):
        co = self.co
        u = torch.zeros(co.tails.K.shape[1], co.tails.K.shape[3], dtype=torch.bool, device="cuda")
        for c, n in enumerate(co.rows.tolist()):
            r = torch.arange(n, device="cuda")
            u[co.tails.table[c].long()[r // 4], r % 4] = True
        return u


def drafts_inputs(m, N, n, seed):
    rng = random.Random(seed)
    chains = [[0], [0, 1, 3, 8], [0, 2, 4, 6, 7], [0, 2, 5], []]
    out = []
    for _ in range(n):
        pick = [rng.choice(chains) for _ in range(N)]
        path = torch.tensor([p + [0] * (9 - len(p)) for p in pick], dtype=torch.int32, device="cuda")
        out.append((m.project(9 * N), path, torch.tensor([len(p) for p in pick], dtype=torch.int32, device="cuda")))
    return out


@pytest.mark.parametrize("two", [False, True])
def test_graph_replays_match_eager_drafts(two):
    # one graph of everything, or one of the draft and one of the rest, which share
    # the workspace; the program's own work and other instances between the replays
    import paper_2609_06663_amd as P
    m = Model(6, "bf16", 2, 28, 4, 128, 4, [1200, 800])
    ep_of = lambda: m.prefill([250, 130], P.PER_HEAD)  # noqa: E731
    state = m.g.get_state()
    eager = Fixed(m, ep_of, [4, 3])
    m.g.set_state(state)
    captured = Fixed(m, ep_of, [4, 3])
    m.g.set_state(state)
    other = Fixed(m, ep_of, [4, 3])
    inputs = drafts_inputs(m, 7, 14, 6)
    want = []
    for i in inputs:
        eager.put(*i)
        eager.draft()
        eager.rest()
        torch.cuda.synchronize()
        want.append(eager.state())
    assert max(eager.co.positions.tolist()) > 1200 + Fixed.LIMIT and max(eager.co.rows.tolist()) <= Fixed.LIMIT
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other.put(*inputs[0])
        other.draft()
        other.rest()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    say("capture")
    graphs = [torch.cuda.CUDAGraph() for _ in range(1 + two)]
    with torch.cuda.graph(graphs[0]):
        captured.draft()
        if not two:
            captured.rest()
    if two:
        with torch.cuda.graph(graphs[1]):
            captured.rest()
    torch.cuda.synchronize()
    for n, i in enumerate(inputs):
        captured.put(*i)
        if n:
            other.put(*i)
            other.draft()
            other.rest()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        say(f"replay {n}")
        for name, a, b, o in zip(("O", "lse", "rows", "positions", "K", "V", "mass", "tail_mass"), captured.state(), want[n], other.state()):
            assert torch.equal(a, b), (n, name)
            assert torch.equal(o, b), (n, name, "eager")


@pytest.mark.parametrize("explicit", [False, True])
def test_drafts_on_a_stream_that_is_not_current(explicit):
    # a wait of some milliseconds before each: what went to another stream would come before
    import paper_2609_06663_amd as P
    m = Model(7, "bf16", 1, 8, 2, 128, 4, [600, 300])
    ep_of = lambda: m.prefill([120, 70], P.PER_HEAD)  # noqa: E731
    state = m.g.get_state()
    eager = Fixed(m, ep_of, [3, 2])
    m.g.set_state(state)
    t = Fixed(m, ep_of, [3, 2])
    inputs = drafts_inputs(m, 5, 8, 7)
    want = []
    for i in inputs:
        eager.put(*i)
        eager.draft()
        eager.rest()
        torch.cuda.synchronize()
        want.append(eager.state())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for n, i in enumerate(inputs):
        with torch.cuda.stream(s):
            torch.cuda._sleep(5_000_000)
            t.put(*i)
            if not explicit:
                t.draft()
                t.rest()
        if explicit:
            t.co.length = 0
            t.co.draft(*t.x, t.tree, stream=s, max_tail=t.MOST)
            t.rest()  # (on the draft's)
        s.synchronize()
        for name, a, b in zip(("O", "lse", "rows", "positions", "K", "V", "mass", "tail_mass"), t.state(), want[n]):
            assert torch.equal(a, b), (n, name)
        torch.cuda.synchronize()


def test_calls_on_several_streams_at_once():
    # with workspaces of their own on four streams: the bits of the same calls alone
    import paper_2609_06663_amd as P
    from test_gpu_evict import masses
    say("four streams")
    trees = [Trees(30 + i, "bf16", 1, 28, 4, 128, [[[3000 + 100 * i]] * 4], [3], [50 + i] * 3, 20 + i) for i in range(4)]
    want = [t.run() for t in trees]
    mass = [(masses("plain", t.g, (t.Kc.shape[0],)), masses("plain", t.g, t.tk.shape[:-1])) for t in trees]
    lone = []
    for t, (m, tm), (O, lse) in zip(trees, mass, want):
        a, b = m.clone(), tm.clone()
        path = torch.arange(t.nodes, dtype=torch.int32, device="cuda").expand(3, -1).contiguous()
        acc = torch.tensor([3, 0, 7], dtype=torch.int32, device="cuda")
        P.ecokv_accumulate(t.Q, lse, t.Kc, t.shape, t.fan, t.counts, t.offsets, t.max_count, t.tails, t.tail_counts, t.max_tail, a, b, path, acc)
        K, V, n = t.Kc.clone(), t.Vc.clone(), t.counts.clone()
        P.ecokv_evict(K, V, t.shape, n, t.offsets, t.max_count, 2000, 1500, 9, a)
        lone.append((path, acc, a, b, K, V, n))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in trees]
    for rep in range(3):
        outs = []
        for t, s, (m, tm), (path, acc, *_) in zip(trees, streams, mass, lone):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                O, lse = torch.zeros((1, 28, 3 * t.nodes, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 28, 3 * t.nodes), device="cuda")
                a, b, K, V, n = m.clone(), tm.clone(), t.Kc.clone(), t.Vc.clone(), t.counts.clone()
            P.ecokv_decode_tree(t.Q, K, V, t.shape, t.fan, n, t.offsets, t.max_count, t.tails, t.tail_counts, t.max_tail, t.masks, O, lse, stream=s)
            P.ecokv_accumulate(t.Q, lse, K, t.shape, t.fan, n, t.offsets, t.max_count, t.tails, t.tail_counts, t.max_tail, a, b, path, acc, stream=s)
            P.ecokv_evict(K, V, t.shape, n, t.offsets, t.max_count, 2000, 1500, 9, a, stream=s)
            outs.append((O, lse, a, b, K, V, n))
        torch.cuda.synchronize()
        for i, (got, w, l) in enumerate(zip(outs, want, lone)):
            for j, (x, y) in enumerate(zip(got, (*w, *l[2:]))):
                assert torch.equal(x, y), (rep, i, j)


def test_pools_past_32_bits():
    """Pools whose last pages lie past 2^32 bytes in K and V, and kept rows past 2^32 bytes."""
    import paper_2609_06663_amd as P
    say("pools past 32 bits")
    t = Masses(21, "bf16", 1, 8, 8, 128, [[[900]] * 8], [2], [200, 137], 6, [3, 6], page=64)
    pages = (2 ** 32 + 2 ** 26) // (8 * 64 * 128 * 2)
    used, first = t.tk.shape[1], pages - t.tk.shape[1]
    K, V = (torch.zeros((1, pages, 8, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[:, first:], V[:, first:] = t.tk, t.tv
    tm = torch.zeros((1, pages, 8, 64), device="cuda")
    tm[:, first:] = t.tail_mass
    rows = (2 ** 32 + 2 ** 26) // 256
    n = t.Kc.shape[0]
    Kc, Vc = (torch.zeros((rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    Kc[rows - n:], Vc[rows - n:] = t.Kc, t.Vc
    mass = torch.zeros(rows, device="cuda")
    mass[rows - n:] = t.mass
    small = [x.clone() for x in (t.Kc, t.Vc, t.mass, t.tk, t.tv, t.tail_mass)]
    far = P.Tails(K, V, t.table + first)
    got = []
    for (kc, vc, m, off), (tails, tmass) in (((small[0], small[1], small[2], t.offsets), (P.Tails(small[3], small[4], t.table), small[5])),
                                             ((Kc, Vc, mass, t.offsets + (rows - n)), (far, tm))):
        counts, tc = t.counts.clone(), t.tail_counts.clone()
        say("commit")
        P.ecokv_commit(t.shape, tails, tc - t.acc_t, t.path_t, t.acc_t)
        say("accumulate")
        P.ecokv_accumulate(t.Q, t.lse, kc, t.shape, t.fan, counts, off, t.max_count, tails, tc, t.max_tail, m, tmass, t.path_t, t.acc_t, 0.5)
        say("evict")
        P.ecokv_evict(kc, vc, t.shape, counts, off, t.max_count, 700, 600, 4, m)
        P.ecokv_evict_tails(t.shape, tails, tc, t.max_tail, 150, 100, 4, tmass)
        torch.cuda.synchronize()
        got.append([kc[-n:], vc[-n:], m[-n:], tails.K[:, -used:], tails.V[:, -used:], tmass[:, -used:], counts, tc])
    for i, (a, b) in enumerate(zip(*got)):
        ints = {torch.bfloat16: torch.int16, torch.float32: torch.int32}.get(a.dtype, a.dtype)
        assert torch.equal(a.contiguous().view(ints), b.contiguous().view(ints)), i
    assert got[0][6].tolist() == [600] * 8 and got[0][7].tolist() == [100, 137]
    assert not bool(Kc[:rows - n].any()) and not bool(K[:, :first].any()) and not bool(tm[:, :first].any())


def test_workspaces_made_by_the_binding():
    import paper_2609_06663_amd as P
    say("no workspace given")
    t = Trees(40, "bf16", 1, 8, 2, 128, [[[300], [200]]], [2], [20, 33], 12)
    O, lse = t.run()
    O2 = torch.empty_like(O)
    P.ecokv_decode_tree(t.Q, t.Kc, t.Vc, t.shape, t.fan, t.counts, t.offsets, t.max_count, t.tails, t.tail_counts, t.max_tail, t.masks, O2)
    torch.cuda.synchronize()
    assert torch.equal(O, O2)
