"""Rows whose step or commit is not followed by accumulated weights, before and after
evictions that moved other rows out of their places: they begin with nothing, and what
is accumulated and evicted later goes by their own weights."""
import sys

import pytest
import torch

from cache_cases import Cache
from test_gpu_drafts import Run, as_case
from test_gpu_evict import Masses, masses

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def say(msg):
    print(f"[gpu-masses] {msg}", file=sys.stderr, flush=True)


@pytest.mark.parametrize("dtype,L,Hkv,D,page,limit,keep,recent,tails", [
    ("bf16", 2, 2, 64, 16, 40, 30, 25, [41, 50, 300, 40, 0, 1]),
    ("f32", 1, 3, 128, 8, 64, 64, 64, [65, 100, 64, 700]),
    ("bf16", 1, 1, 64, 64, 5, 1, 0, [900, 2, 6]),
    ("f32", 1, 2, 64, 4, 600, 300, 290, [601, 2100, 9000]),    # (more rows than registers hold keys)
])
def test_places_that_an_eviction_empties(dtype, L, Hkv, D, page, limit, keep, recent, tails):
    import paper_2609_06663_amd as P
    say(f"{dtype} {L} {Hkv} {D}: {tails} -> {keep} of more than {limit}")
    t = Cache(12, dtype, L, Hkv, Hkv, D, [[[1]] * Hkv] * L, [len(tails)], tails, page=page)
    mass = masses("plain", t.g, t.tk.shape[:-1])
    before = mass.clone()
    P.ecokv_evict_tails(t.shape, t.tails, t.tail_counts, t.max_tail, limit, keep, recent, mass)
    torch.cuda.synchronize()
    other = torch.ones(mass.shape[1], page, dtype=torch.bool, device="cuda")
    for c, n in enumerate(tails):
        p, r = t.tail_index(c, list(range(n)))
        other[p, r] = False
        got, was = mass[:, p, :, r], before[:, p, :, r]     # [rows][L][Hkv]
        if n > limit:
            assert bool((got[keep:] == 0).all()) and bool((got[:keep] > 0).all())
        else:
            assert torch.equal(got, was)
    assert torch.equal(mass.transpose(1, 2)[:, :, other], before.transpose(1, 2)[:, :, other])


def evicted_run():
    """Past an eviction that leaves rows behind every tail."""
    run = Run(2, "bf16", 2, 8, 2, 128, 4, [300, 200], [60, 40], "per_head", [2, 1], 4, 40, 8)
    for _ in range(12):
        run.step()
    run.evict(11, 5, 1)
    assert run.co.rows.tolist() == [5] * 3
    return run


def mass_of(co, rows):
    """[N][rows][L][Hkv] of rows of every tail."""
    t = as_case(Cache, co)
    return torch.stack([co.tail_mass[:, p, :, r] for p, r in (t.tail_index(c, rows) for c in range(co.fan[-1]))])


def project_step(run):
    run.co.step(*run.m.project(3))


def project_draft(run, parents, accepted):
    co = run.co
    co.draft(*run.m.project(3 * len(parents)), co.tree(parents))
    path = torch.arange(len(parents), dtype=torch.int32, device="cuda").expand(3, -1).contiguous()
    co.commit(path, torch.full((3,), accepted, dtype=torch.int32, device="cuda"))
    co.length = int(co.rows.max())


@pytest.mark.parametrize("how", ["steps", "drafts"])
def test_rows_that_were_not_weighed(how):
    say(f"skipped: {how}")
    run = evicted_run()
    co = run.co
    if how == "steps":
        for _ in range(3):
            project_step(run)
            co.advance()
    else:
        project_draft(run, [-1, 0, 1, 2], 3)
    torch.cuda.synchronize()
    assert co.rows.tolist() == [8] * 3 and bool((mass_of(co, [5, 6, 7]) == 0).all())
    run.step()        # (weighed, and checked against 64 bits)
    now = mass_of(co, [5, 6, 7, 8])
    assert bool((now > 0).all())
    # the weights of that step alone
    t = as_case(Masses, co, Q=co.Q_dec, lse=co.lse, M=1, path=[[0]] * 3, acc=[1] * 3)
    for l in range(2):
        for h in range(2):
            for c in range(3):
                p, r = t.tail_index(c, [5, 6, 7, 8])
                x = co.Q_dec[l, 4 * h:4 * h + 4, c].double() @ co.tails.K[l, p, h, r].double().t() / 128 ** 0.5 - co.lse[l, 4 * h:4 * h + 4, c, None].double()
                want = x.exp().sum(0)
                assert bool(((now[c, :, l, h].double() - want).abs() <= 2.0 ** -10 * want).all())


def test_an_eviction_right_after_rows_that_were_not_weighed():
    say("evicted unweighed")
    run = evicted_run()
    co = run.co
    heavy = mass_of(co, list(range(5)))
    assert bool((heavy > 0).all())
    project_draft(run, [-1] * 4, 4)
    kept = co.tails.K[:, co.tails.table.long()][:, :, :, :, :].clone()
    run.evict(8, 5, 0)      # (nine rows; the five that were weighed stay where they are)
    assert co.rows.tolist() == [5] * 3 and torch.equal(mass_of(co, list(range(5))), heavy)
    t, u = kept, co.tails.K[:, co.tails.table.long()]
    assert torch.equal(t[:, :, 0], u[:, :, 0])     # (a page of four rows)


@pytest.mark.parametrize("then", ["step", "draft"])
def test_a_step_that_was_weighed_and_replaced(then):
    say(f"replaced by a {then}")
    run = evicted_run()
    co = run.co
    project_step(run)
    co.accumulate()
    assert bool((mass_of(co, [5]) > 0).all())
    old = mass_of(co, list(range(5)))
    if then == "step":
        project_step(run)
        co.advance()
    else:
        project_draft(run, [-1, -1], 1)
    torch.cuda.synchronize()
    assert co.rows.tolist() == [6] * 3 and bool((mass_of(co, [5, 6]) == 0).all()) and torch.equal(mass_of(co, list(range(5))), old)
    # one that was not replaced keeps what it got
    project_step(run)
    co.accumulate()
    got = mass_of(co, [6])
    co.advance()
    project_step(run)
    co.advance()
    torch.cuda.synchronize()
    assert bool((got > 0).all()) and torch.equal(mass_of(co, [6]), got) and bool((mass_of(co, [7]) == 0).all())


def test_graphs_with_and_without_weights():
    """A captured step without weights, one with them, and an eviction, replayed in any order."""
    say("captured")
    run = evicted_run()
    co, m = run.co, run.m
    x = [t.clone() for t in m.project(3)]

    def token(weighed):
        co.length = 0
        co.step(*x, max_tail=40)
        co.advance()
        if weighed:
            co.accumulate(max_tail=40)
        else:
            co._unweighed = None

    torch.cuda.synchronize()
    graphs = {}
    for name, f in (("bare", lambda: token(False)), ("weighed", lambda: token(True)), ("evict", lambda: co.evict(11, 5, 1, max_tail=40))):
        graphs[name] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[name]):
            f()
    for turn in range(3):
        say(f"replays {turn}")
        n = int(co.rows.max())
        assert n == 5
        for i, name in enumerate(["weighed", "bare", "weighed", "bare", "bare", "bare", "weighed"]):
            for d, s in zip(x, m.project(3)):
                d.copy_(s)
            graphs[name].replay()
            torch.cuda.synchronize()
            now = mass_of(co, [n + i])
            assert co.rows.tolist() == [n + i + 1] * 3 and bool((now > 0).all() if name == "weighed" else (now == 0).all()), (turn, i)
        graphs["evict"].replay()
        torch.cuda.synchronize()
        assert bool((mass_of(co, list(range(5, 12))) == 0).all())
