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
