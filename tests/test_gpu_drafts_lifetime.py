"""Trees, paths and numbers of accepted nodes that the program drops as soon as a call
has returned, on the stream that it enqueued the work on and on another, and trees of
captured graphs: what is allocated next does not change what the calls read."""
import sys

import pytest
import torch

from test_gpu_drafts import drafts_inputs
from test_gpu_generate import Model

pytestmark = pytest.mark.gpu

PARENTS = [-1, 0, 0, 1, 2, 2, 4, 6, 3]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-drafts] {msg}", file=sys.stderr, flush=True)


def both():
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    m = Model(8, "bf16", 1, 8, 2, 128, 4, [600, 300])
    ep = m.prefill([120, 70], P.PER_HEAD)
    return m, [Continuations(ep, [3, 2], 40, m.rope, 4, 9, True) for _ in range(2)]


def state(co):
    # (rows behind a tail were never written)
    mine = torch.arange(co.tails.table.shape[1] * 4, device="cuda") < co.rows[:, None]
    tails = [torch.where(mine[None, :, None, :, None], x[:, co.tails.table.long()].transpose(2, 3).flatten(3, 4), 0) for x in (co.tails.K, co.tails.V)]
    return [t.clone() for t in (co.O_nodes, co.lse_nodes, co.rows, co.positions, co.mass, *tails)]


def overwrite():
    """What the sizes of trees, paths and counts would be given again, in other values."""
    return [torch.full((n,), 77, dtype=t, device="cuda") for n in (5, 45, 90) for t in (torch.int32, torch.int64) for _ in range(8)]


@pytest.mark.parametrize("explicit", [False, True])
def test_dropped_trees_and_paths(explicit):
    m, (a, b) = both()
    s = torch.cuda.Stream()
    junk = []
    for i, (x, path, acc) in enumerate(drafts_inputs(m, 5, 5, 3)):
        say(f"dropped trees, draft {i}")
        a.draft(*x, a.tree(PARENTS))
        a.commit(path, acc)
        a.accumulate(0.9)
        torch.cuda.synchronize()
        want = state(a)
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
        if explicit:
            b.draft(*x, b.tree(PARENTS), stream=s)
        else:
            tree = b.tree(PARENTS)
            with torch.cuda.stream(s):
                b.draft(*x, tree)
            del tree
        junk.append(overwrite())
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
        p, n = path.clone(), acc.clone()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            b.commit(p, n)
            b.accumulate(0.9)
        del p, n
        b._unweighed = None
        junk.append(overwrite())
        torch.cuda.synchronize()
        for j, (y, z) in enumerate(zip(state(b), want)):
            assert torch.equal(y, z), (i, j)
        a.length = b.length = int(a.rows.max())


def test_trees_of_captured_graphs():
    m, (a, b) = both()
    inputs = drafts_inputs(m, 5, 6, 4)
    static = [t.clone() for t in (*inputs[0][0], *inputs[0][1:])]

    def turn(co, x, path, acc, tree):
        co.length = 0
        co.draft(*x, tree, max_tail=36)
        co.commit(path, acc)
        co.accumulate(0.9, max_tail=36)

    say("capture")
    graph = torch.cuda.CUDAGraph()
    tree = b.tree(PARENTS)  # (a copy from the host: before the capture)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        turn(b, static[:3], *static[3:], tree)
    del tree
    junk = [overwrite()]
    for i, (x, path, acc) in enumerate(inputs):
        say(f"replay {i}")
        for d, v in zip(static, (*x, path, acc)):
            d.copy_(v)
        turn(a, x, path, acc, a.tree(PARENTS))
        graph.replay()
        torch.cuda.synchronize()
        junk.append(overwrite())
        for j, (y, z) in enumerate(zip(state(b), state(a))):
            assert torch.equal(y, z), (i, j)
