"""Commits that leave a continuation as it is (numbers out of their bounds, paths that
do not ascend, rows without a page): ecokv_commit says so, and a program's counters,
positions and masses go on as if nothing had been accepted there."""
import sys

import pytest
import torch

from test_gpu_drafts import Run, as_case
from test_gpu_evict import Masses
from test_gpu_tree import Trees

pytestmark = pytest.mark.gpu

NODES = 6
# accepted, path: what is taken
TAKES = [(3, [0, 2, 5, 9, 9, 9], 3), (3, [2, 1, 4, 0, 0, 0], 0), (2, [1, 1, 2, 3, 4, 5], 0), (7, [0, 1, 2, 3, 4, 5], 0), (-1, [0, 1, 2, 3, 4, 5], 0),
         (2, [-1, 3, 0, 0, 0, 0], 0), (2, [4, 6, 0, 0, 0, 0], 0), (0, [3, 2, 1, 0, 9, -9], 0), (6, [0, 1, 2, 3, 4, 5], 6), (1, [5, 0, 0, 0, 0, 0], 1),
         (2, [3, 2 ** 31 - 1, 0, 0, 0, 0], 0), (-2 ** 31, [0, 1, 2, 3, 4, 5], 0)]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-commit] {msg}", file=sys.stderr, flush=True)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,L,Hkv,D", [("bf16", 3, 4, 128), ("f32", 1, 1, 64)])
def test_what_was_taken(dtype, L, Hkv, D):
    import paper_2609_06663_amd as P
    say(f"taken {dtype} {L} {Hkv} {D}")
    N = len(TAKES) + 3
    tails = [5 + 3 * c for c in range(N)]
    t = Trees(41, dtype, L, Hkv, Hkv, D, [[[1]] * Hkv] * L, [N], tails, NODES, page=4)
    accepted, path, want = (list(v) for v in zip(*TAKES, *[(2, [0, 4, 0, 0, 0, 0], 0)] * 3))
    # a count below 0; no page for a row that goes, and for the place of one
    t.tail_counts[N - 3] = -1
    t.table[N - 2, (tails[N - 2] + 4) // 4] = -1
    t.table[N - 1, tails[N - 1] // 4] = t.tk.shape[1]
    taken = torch.full((N + 2,), -7, dtype=torch.int32, device="cuda")
    K, V = t.tk.clone(), t.tv.clone()
    P.ecokv_commit(t.shape, t.tails, t.tail_counts, i32(path), i32(accepted), taken=taken)
    torch.cuda.synchronize()
    assert taken.tolist() == want + [-7, -7]
    # the same rows as without it
    K2, V2 = t.tk.clone(), t.tv.clone()
    t.tk.copy_(K), t.tv.copy_(V)
    P.ecokv_commit(t.shape, t.tails, t.tail_counts, i32(path), i32(accepted))
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(K2.view(bits), t.tk.view(bits)) and torch.equal(V2.view(bits), t.tv.view(bits))
    assert not torch.equal(K.view(bits), K2.view(bits))


def test_a_program_goes_on_without_what_was_refused():
    say("refused paths")
    run = Run(3, "bf16", 2, 8, 2, 128, 4, [300, 200], [60, 40], "per_head", [6, 6], 4, 60, NODES)
    co = run.co
    for _ in range(5):
        run.step()
    assert len(TAKES) == co.fan[-1]
    accepted, path, want = zip(*TAKES)
    parents = [-1, 0, 0, 1, 2, 2]
    co.draft(*run.m.project(12 * NODES), co.tree(parents))
    before, masses = co.tail_mass.clone(), co.mass.clone()
    p, a = i32(path), i32(accepted)
    co.commit(p, a)
    torch.cuda.synchronize()
    assert co.rows.tolist() == [5 + n for n in want] and co.tail_counts.tolist() == [6 + n for n in want]
    assert co.positions.tolist() == [305 + n for n in want[:6]] + [205 + n for n in want[6:]]
    assert a.tolist() == list(accepted)
    # the weights of what was taken, and of nothing else
    t = as_case(Masses, co, Q=co.Q_nodes, lse=co.lse_nodes, M=NODES, path=[list(v[:n]) for v, n in zip(path, want)], acc=list(want), mass=masses,
                tail_mass=before)
    co.accumulate(0.9)
    t.check(co.mass, co.tail_mass, 0.9)
    co.length = int(co.rows.max())
    run.step()
    run.draft()


def test_numbers_of_another_shape_are_refused():
    run = Run(4, "f32", 1, 2, 1, 64, 4, [60], [20], "per_head", [2], 4, 20, 2)
    co = run.co
    co.draft(*run.m.project(4), co.tree([-1, 0]))
    p = i32([[0, 1]] * 2)
    for bad in (i32([[1], [1]]), i32([1, 1, 1]), i32([1]), i32(1)):
        with pytest.raises(ValueError, match="accepted has shape"):
            co.commit(p, bad)
    for bad in ([1, 1], None):
        with pytest.raises(TypeError, match="accepted"):
            co.commit(p, bad)
    torch.cuda.synchronize()
    assert co.rows.tolist() == [0, 0] and co.length == 0
    co.commit(p, i32([1, 2]))
    torch.cuda.synchronize()
    assert co.rows.tolist() == [1, 2]
