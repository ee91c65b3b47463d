"""pipeline.Continuations and the handles of its calls on the GPU: streams given
to steps, tensors of Rope and Tails replaced between calls, arguments that a call
does not read."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-continuations] {msg}", file=sys.stderr, flush=True)


@pytest.mark.parametrize("explicit", [False, True])
def test_steps_on_a_stream_that_is_not_current(explicit):
    # every step waits on its stream for some milliseconds of other work, so that an
    # increment of the counters anywhere else would come before it
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    from test_gpu_generate import Model
    m = Model(60, "bf16", 1, 28, 4, 128, 4, [600, 300])
    ep = m.prefill([120, 70], P.PER_HEAD)
    steps = [m.project(5) for _ in range(4)]
    eager, co = Continuations(ep, [3, 2], 4, m.rope, 2), Continuations(ep, [3, 2], 4, m.rope, 2)
    want = []
    for x in steps:
        eager.step(*x)
        want.append((eager.O.clone(), eager.lse.clone(), eager.Q_dec.clone()))
        eager.advance()
    torch.cuda.synchronize()
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    say(f"steps on a stream of their own, advance {'on the same' if explicit else 'without a stream'}")
    with torch.cuda.stream(other):
        for x in steps:
            with torch.cuda.stream(s):
                torch.cuda._sleep(5_000_000)
            co.step(*x, stream=s)
            with torch.cuda.stream(s):
                got.append((co.O.clone(), co.lse.clone(), co.Q_dec.clone()))
            if explicit:
                co.advance(stream=s)
            else:
                co.advance()
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        for name, x, y in zip(("O", "lse", "Q_dec"), a, b):
            assert torch.equal(x, y), (i, name)
    assert torch.equal(co.tails.K, eager.tails.K) and torch.equal(co.tails.V, eager.tails.V)
    assert co.rows.tolist() == [4] * 5 and co.length == 4


def test_tensors_of_the_handles_replaced_between_calls():
    # a larger pool and table, other frequencies and norms: the next call reads those;
    # the old ones are overwritten first, as memory that was given out again would be
    import paper_2609_06663_amd as P
    from test_gpu_rope import near, turned
    from test_gpu_shared import Case
    c = Case(61, "bf16", 1, 8, 2, 128, [[[300], [200]]], [3], [40, 1, 33], 16)
    O, lse = c.run()
    say("pool and table replaced")
    pages, most = c.tk.shape[1], c.table.shape[1]
    tk, tv = (torch.full_like(t, float("nan")) for t in (c.tk, c.tv))
    t = P.Tails(tk, tv, torch.full_like(c.table, -1))
    got, gl = torch.empty_like(O), torch.empty_like(lse)
    call = lambda: P.ecokv_decode_shared(c.Q, c.Kc, c.Vc, c.shape, c.fan, c.counts, c.offsets, c.max_count, t, c.tail_counts, c.max_tail, got, gl)
    call()
    assert bool(got.isnan().all())
    big = [torch.zeros(1, pages + 9, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.full((3, most + 2), -1, dtype=torch.int32, device="cuda")
    table[:, :most] = c.table + 9
    for b, s in zip(big, (c.tk, c.tv)):
        b[:, 9:] = s
    t.table, (t.K, t.V) = table, big
    call()
    torch.cuda.synchronize()
    assert torch.equal(got, O) and torch.equal(gl, lse)
    say("frequencies and norms replaced")
    g = torch.Generator(device="cuda").manual_seed(62)
    K = torch.randn(1, 37, 2, 128, generator=g, device="cuda").bfloat16()
    w = (1 + 0.1 * torch.randn(128, generator=g, device="cuda")).bfloat16()
    f = [torch.rand(64, generator=g, device="cuda") for _ in range(2)]
    shape, out = P.Shape(1, 4, 2, 128, 4, [0, 37]), torch.empty_like(K)
    r = P.Rope(128, f[0])
    for freq, norm in ((f[0], None), (f[1], None), (f[1], w), (f[0], None)):
        r.freq, r.k_norm = freq, norm
        P.ecokv_prefill_rope(None, K, shape, r, None, None, out)
        near(out, *turned(K, torch.arange(37, device="cuda"), freq, 128, False, 1.0, norm, 1e-6), "bf16")


def test_bounds_past_32_bits_are_refused():
    import paper_2609_06663_amd as P
    from test_gpu_shared import Case
    c = Case(63, "f32", 1, 4, 2, 64, [[[30], [40]]], [2], [5, 6], 16)
    O, lse = torch.empty(1, 4, 2, 64, device="cuda"), torch.empty(1, 4, 2, device="cuda")
    t, ws = P.Tails(c.tk, c.tv, c.table), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for mc, mt, fan in ((2 ** 32 + 40, 6, c.fan), (40, 2 ** 32, c.fan), (40, 6, [0, 2 ** 32 + 2])):
        with pytest.raises(ValueError, match="32 bits"):
            P.ecokv_decode_shared(c.Q, c.Kc, c.Vc, c.shape, fan, c.counts, c.offsets, mc, t, c.tail_counts, mt, O, lse, ws)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_what_a_bound_of_zero_leaves_unread_may_be_empty(dtype, D):
    # the cache of prompts of which nothing was kept, the counts of tails not yet begun
    import paper_2609_06663_amd as P
    from test_gpu_shared import Case
    c = Case(64, dtype, 1, 4, 2, D, [[[30], [0]]], [2], [5, 6], 16)
    O, lse = torch.empty(1, 4, 2, D, device="cuda"), torch.empty(1, 4, 2, device="cuda")
    none, no_counts = c.Kc[:0], c.counts[:0]
    say(f"{dtype} D={D}: nothing kept")
    P.ecokv_decode_shared(c.Q, none, none, c.shape, c.fan, no_counts, no_counts, 0, P.Tails(c.tk, c.tv, c.table), c.tail_counts, 6, O, lse)
    want = c.run(max_count=0)
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    say(f"{dtype} D={D}: no tails")
    P.ecokv_decode_shared(c.Q, c.Kc, c.Vc, c.shape, c.fan, c.counts, c.offsets, 30, None, no_counts, 0, O, lse)
    want = c.run(max_tail=0)
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    say(f"{dtype} D={D}: neither")
    P.ecokv_decode_shared(c.Q, none, none, c.shape, c.fan, no_counts, no_counts, 0, None, no_counts, 0, O, lse)
    assert bool((O == 0).all()) and bool((lse == -float("inf")).all())
