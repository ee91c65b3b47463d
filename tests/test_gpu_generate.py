"""Generation from compressed prompts as a program does it: projections ->
ecokv_prefill_rope -> ecokv_prefill_write -> score, select, compact -> steps of
ecokv_append and ecokv_decode_shared (pipeline.Continuations), against attention
in 64 bits over what the cache and the tails hold; captured in a HIP graph and
replayed; on several streams at once."""
import sys

import pytest
import torch

from test_gpu_rope import near, turned

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-generate] {msg}", file=sys.stderr, flush=True)


class Model:
    """Projections of random numbers: everything of a prompt and of new tokens side by side."""

    def __init__(self, seed, dtype, L, Hq, Hkv, D, w, lens, norm=True, rot=None):
        import paper_2609_06663_amd as P
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.dims, self.dtype, self.lens = (L, Hq, Hkv, D, w), TYPES[dtype], lens
        self.cu = [0]
        for t in lens:
            self.cu.append(self.cu[-1] + t)
        rot = D if rot is None else rot
        freq, factor = P.ecokv_rope_freqs(rot, 10000.0, P.ROPE_BY_PARTS, 4.0, 4096.0)
        self.freq = torch.tensor(freq, device="cuda")
        wt = [(1 + 0.1 * torch.randn(D, generator=self.g, device="cuda")).to(self.dtype) if norm else None for _ in range(2)]
        self.rope = P.Rope(rot, self.freq, factor=factor, q_norm=wt[0], k_norm=wt[1])
        self.params = (rot, False, factor, *wt)
        self.shape = P.Shape(L, Hq, Hkv, D, w, self.cu)

    def project(self, n):
        L, Hq, Hkv, D, _ = self.dims
        x = torch.randn((L, n, Hq + 2 * Hkv, D), generator=self.g, device="cuda").to(self.dtype)
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]

    def prefill(self, budget, mode):
        """The compressed prompts: an EvictionPass, and the rotated keys it read."""
        import paper_2609_06663_amd as P
        from paper_2609_06663_amd.pipeline import EvictionPass
        L, Hq, Hkv, D, w = self.dims
        n, B, R = self.cu[-1], len(self.lens), Hq // Hkv * w
        e = lambda *s, dtype=self.dtype: torch.empty(s, dtype=dtype, device="cuda")
        Q, K, V = self.project(n)
        K_new, Q_win = e(L, n, Hkv, D), e(L, Hq, B, w, D)
        P.ecokv_prefill_rope(Q, K, self.shape, self.rope, None, None, K_new, Q_win)
        Kc, Vc, pre = e(L, Hkv, n, D), e(L, Hkv, n, D), e(L * Hkv * B, 2 * D + 2 * R, dtype=torch.float32)
        P.ecokv_prefill_write(K_new, V.contiguous(), Q_win, self.shape, None, Kc, Vc, pre)
        ep = EvictionPass(self.shape, budget, mode, None, self.dtype)
        ep.run(Kc, Vc, Q_win, pre=pre)
        ep.check()
        own = torch.cat([torch.arange(t, device="cuda") for t in self.lens])
        rot, inter, factor, qw, kw = self.params
        name = "bf16" if self.dtype == torch.bfloat16 else "f32"
        near(K_new, *turned(K, own, self.freq, rot, inter, factor, kw, 1e-6), name)
        q, qs = turned(Q, own, self.freq, rot, inter, factor, qw, 1e-6)
        for s, end in enumerate(self.cu[1:]):
            near(Q_win[:, :, s], q[:, end - w:end].transpose(1, 2), qs[:, end - w:end].transpose(1, 2), name)
        return ep


def check_step(m, co, fan_out, K, V):
    """O and lse of the last step in 64 bits, from the kept rows, the tails and Q_dec; the tails' newest rows."""
    L, Hq, Hkv, D, _ = m.dims
    G, B, page = Hq // Hkv, len(fan_out), co.tails.K.shape[3]
    ep, parent = co.ep, [s for s, f in enumerate(fan_out) for _ in range(f)]
    rot, inter, factor, _, kw = m.params
    name = "bf16" if m.dtype == torch.bfloat16 else "f32"
    n = co.length + 1
    k, ks = turned(K, torch.tensor([m.lens[s] + n - 1 for s in parent], device="cuda"), m.freq, rot, inter, factor, kw, 1e-6)
    for l in range(L):
        for h in range(Hkv):
            for c, s in enumerate(parent):
                u = (l * Hkv + h) * B + s
                o, cnt = int(ep.offsets[u]), int(ep.counts[u])
                pages = co.tails.table[c, :-(-n // page)].long()
                tk, tv = (t[l, pages, h].reshape(-1, D)[:n] for t in (co.tails.K, co.tails.V))
                near(tk[-1], k[l, c, h], ks[l, c, h], name)
                assert torch.equal(tv[-1], V[l, c, h])
                Ks, Vs = torch.cat([ep.Kc[o:o + cnt], tk]).double(), torch.cat([ep.Vc[o:o + cnt], tv]).double()
                q = co.Q_dec[l, h * G:(h + 1) * G, c].double()
                x = q @ Ks.t() / D ** 0.5
                # (the tolerance of tests/test_gpu_shared.py)
                dx = 40 * 2.0 ** -24 * float((q.abs() @ Ks.abs().t()).max()) / D ** 0.5
                err = float((co.O[l, h * G:(h + 1) * G, c].double() - x.softmax(1) @ Vs).abs().max())
                assert err <= (2 * dx + 2.0 ** -18) * float(Vs.abs().max()), (l, h, c, err)
                assert bool(((co.lse[l, h * G:(h + 1) * G, c].double() - x.logsumexp(1)).abs() <= dx + 2.0 ** -20 * 20).all())


@pytest.mark.parametrize("dtype,L,Hq,Hkv,D,w,lens,budget,mode,fan_out,page", [
    ("bf16", 2, 28, 4, 128, 4, [1500, 700], [300, 100], "per_head", [3, 2], 4),
    ("bf16", 1, 8, 8, 64, 8, [900], [200], "per_head", [5], 16),
    ("bf16", 1, 16, 4, 128, 4, [400, 3001, 60], [80, 500, 60], "flat", [1, 0, 4], 2),
    ("f32", 2, 4, 2, 64, 4, [500], [[100, 40], [20, 300]], "heads", [2], 1),
])
def test_generation(dtype, L, Hq, Hkv, D, w, lens, budget, mode, fan_out, page):
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    say(f"{dtype} {L} layers {Hq}/{Hkv} heads of {D}: prompts {lens} -> {budget} ({mode}), continuations {fan_out}")
    m = Model(1, dtype, L, Hq, Hkv, D, w, lens)
    ep = m.prefill(budget, {"per_head": P.PER_HEAD, "flat": P.LAYER_FLAT, "heads": P.HEAD_BUDGETS}[mode])
    co = Continuations(ep, fan_out, 7, m.rope, page)
    assert int(ep.counts.max()) <= co.max_count
    for _ in range(7):
        Q, K, V = m.project(co.fan[-1])
        co.step(Q, K, V)
        check_step(m, co, fan_out, K, V)
        co.advance()
    with pytest.raises(ValueError, match="hold 7"):
        co.step(Q, K, V)
    with pytest.raises(ValueError, match="each prompt"):
        Continuations(ep, fan_out + [1], 7, m.rope)
    with pytest.raises(ValueError, match="no continuation"):
        Continuations(ep, [0] * len(lens), 7, m.rope)
    with pytest.raises(ValueError, match="max_new"):
        Continuations(ep, fan_out, 0, m.rope)


def test_graph_replays_match_eager_steps():
    # one captured step, replayed: each replay appends where the device's counters
    # stand, and must give the bits of the eager step on the same projections
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    m = Model(2, "bf16", 2, 28, 4, 128, 4, [1200, 800])
    ep = m.prefill([250, 130], P.PER_HEAD)
    steps = [m.project(7) for _ in range(6)]
    eager = Continuations(ep, [4, 3], 6, m.rope, 4)
    want = []
    for x in steps:
        eager.step(*x, max_tail=6)
        torch.cuda.synchronize()
        want.append((eager.O.clone(), eager.lse.clone(), eager.Q_dec.clone()))
        eager.advance()
    co, other = Continuations(ep, [4, 3], 6, m.rope, 4), Continuations(ep, [4, 3], 6, m.rope, 4)
    static = [t.clone() for t in steps[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other.step(*static, max_tail=6)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    say("capture")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        co.step(*static, max_tail=6)
        co.advance()
    torch.cuda.synchronize()
    for i, x in enumerate(steps):
        for dst, src in zip(static, x):
            dst.copy_(src)
        other.step(*x, max_tail=6)  # the program's own work between replays
        other.advance()
        g.replay()
        torch.cuda.synchronize()
        say(f"replay {i}")
        for name, a, b in zip(("O", "lse", "Q_dec"), (co.O, co.lse, co.Q_dec), want[i]):
            assert torch.equal(a, b), (i, name)
        assert torch.equal(other.O, want[i][0])
    for t, u in ((co.tails.K, eager.tails.K), (co.tails.V, eager.tails.V)):
        # six tokens of each: a whole page and two rows of the next; nobody wrote the rest
        assert torch.equal(t[:, 0::2], u[:, 0::2]) and torch.equal(t[:, 1::2, :, :2], u[:, 1::2, :, :2])
    assert co.rows.tolist() == [6] * 7


def test_graph_replays_of_prompts_and_of_large_splits():
    # prefill_rope and decode_shared captured on shapes that take the wide tiles and
    # the many-partial merge; inputs change between replays
    import paper_2609_06663_amd as P
    from test_gpu_shared import Case
    m = Model(3, "bf16", 1, 28, 4, 128, 4, [2000])
    c = Case(18, "bf16", 1, 28, 4, 128, [[[6553]] * 4], [20], [100 + 9 * i for i in range(20)], 16)
    c.max_count = 3_000_000
    L, Hq, Hkv, D, w = m.dims
    e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
    Q, K, V = (t.contiguous() for t in m.project(2000))
    Q2, K2, _ = m.project(2000)
    Ko, Qw, O, lse = e(L, 2000, Hkv, D), e(L, Hq, 1, w, D), e(1, 28, 20, 128, dtype=torch.float32), e(1, 28, 20, dtype=torch.float32)
    ws = torch.empty(P.ecokv_decode_shared_workspace_size(c.shape, c.fan, c.max_count, c.max_tail), dtype=torch.uint8, device="cuda")
    tails = P.Tails(c.tk, c.tv, c.table)

    def work():
        P.ecokv_prefill_rope(Q, K, m.shape, m.rope, None, None, Ko, Qw)
        P.ecokv_decode_shared(c.Q, c.Kc, c.Vc, c.shape, c.fan, c.counts, c.offsets, c.max_count, tails, c.tail_counts, c.max_tail, O, lse, ws)

    inputs = [(Q.clone(), K.clone(), c.Q.clone()), (Q2.clone(), K2.clone(), torch.randn_like(c.Q))]
    want = []
    for a in inputs:
        for d, s in zip((Q, K, c.Q), a):
            d.copy_(s)
        work()
        torch.cuda.synchronize()
        want.append([t.clone() for t in (Ko, Qw, O, lse)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work()
    for rep, which in enumerate([0, 1, 1, 0, 1]):
        for d, s in zip((Q, K, c.Q), inputs[which]):
            d.copy_(s)
        for t in (Ko, Qw, O, lse):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        say(f"replay {rep} on input {which + 1}")
        assert all(torch.equal(a, b) for a, b in zip((Ko, Qw, O, lse), want[which])), rep


def test_calls_on_several_streams_at_once():
    # four calls with workspaces of their own on four streams, given by the argument
    # and as the current one: the bits of the same calls one after another
    import paper_2609_06663_amd as P
    from test_gpu_shared import Case
    cases = [Case(30 + i, "bf16", 1, 28, 4, 128, [[[3000 + 100 * i]] * 4], [8 + i], [50 + i] * (8 + i), 16) for i in range(4)]
    want = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = []
    torch.cuda.synchronize()
    for rep in range(3):
        for i, (c, s) in enumerate(zip(cases, streams)):
            O, lse = torch.zeros_like(want[i][0]), torch.zeros_like(want[i][1])
            s.wait_stream(torch.cuda.current_stream())
            args = (c.Q, c.Kc, c.Vc, c.shape, c.fan, c.counts, c.offsets, c.max_count, P.Tails(c.tk, c.tv, c.table), c.tail_counts, c.max_tail, O, lse)
            if i % 2:
                with torch.cuda.stream(s):
                    P.ecokv_decode_shared(*args)
            else:
                P.ecokv_decode_shared(*args, stream=s)
            outs.append((i, O, lse))
    torch.cuda.synchronize()
    for i, O, lse in outs:
        assert torch.equal(O, want[i][0]) and torch.equal(lse, want[i][1]), i


def test_two_graphs_share_a_workspace():
    # graphs of different splits over one workspace, replayed in order on one
    # stream with an eager call of the same workspace between them
    import paper_2609_06663_amd as P
    from test_gpu_shared import Case
    cases = [Case(40, "bf16", 1, 28, 4, 128, [[[6553]] * 4], [8], [200] * 8, 64),
             Case(41, "f32", 1, 8, 2, 64, [[[300, 77]] * 2], [3, 1], [20, 0, 5, 33], 4)]
    sizes = [P.ecokv_decode_shared_workspace_size(c.shape, c.fan, c.max_count, c.max_tail) for c in cases]
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    want = [c.run() for c in cases]
    outs = [(torch.empty_like(o), torch.empty_like(l)) for o, l in want]
    tails = [P.Tails(c.tk, c.tv, c.table) for c in cases]

    def work(i):
        c = cases[i]
        P.ecokv_decode_shared(c.Q, c.Kc, c.Vc, c.shape, c.fan, c.counts, c.offsets, c.max_count, tails[i], c.tail_counts, c.max_tail, *outs[i], ws)

    graphs = []
    for i in range(2):
        work(i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            work(i)
    for rep in range(4):
        for o, l in outs:
            o.zero_(), l.zero_()
        graphs[rep % 2].replay()
        work(1 - rep % 2)
        say(f"round {rep}")
        torch.cuda.synchronize()
        graphs[1 - rep % 2].replay()
        torch.cuda.synchronize()
        for (o, l), (wo, wl) in zip(outs, want):
            assert torch.equal(o, wo) and torch.equal(l, wl), rep


def test_a_workspace_made_by_the_binding_is_in_order_with_its_stream(monkeypatch):
    # allocated and filled on the call's stream, whatever the current one is
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd import ecokv as E
    from test_gpu_shared import Case
    c = Case(50, "bf16", 1, 8, 2, 128, [[[900], [400]]], [3], [20, 0, 5], 16)
    O, lse = c.run()
    seen, zeros = [], torch.zeros
    monkeypatch.setattr(E.torch, "zeros", lambda *a, **k: (seen.append(torch.cuda.current_stream()), zeros(*a, **k))[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    O2, lse2 = torch.empty_like(O), torch.empty_like(lse)
    tails = P.Tails(c.tk, c.tv, c.table)
    call = lambda **kw: P.ecokv_decode_shared(c.Q, c.Kc, c.Vc, c.shape, c.fan, c.counts, c.offsets, c.max_count, tails, c.tail_counts, c.max_tail,
                                              O2, lse2, **kw)
    call(stream=s)
    s.synchronize()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    call()
    torch.cuda.synchronize()
    assert seen == [s, torch.cuda.current_stream()]
