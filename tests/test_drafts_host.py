"""pipeline.Continuations with drafts, masses and evictions on the host: the order
of its calls, what it gives them, and which it refuses.  The library's calls are
replaced by recorders, the tensors are the CPU's."""
import pytest
import torch

from test_continuations_host import Recorder


@pytest.fixture
def rec(monkeypatch):
    from paper_2609_06663_amd import pipeline
    r = Recorder(monkeypatch)
    for name in ("ecokv_append", "ecokv_decode_shared", "ecokv_decode_tree", "ecokv_commit", "ecokv_accumulate", "ecokv_evict", "ecokv_evict_tails"):
        def call(*a, _name=name[6:], **k):
            r.calls.append((_name, [x.clone() if isinstance(x, torch.Tensor) else x for x in a], k))
        monkeypatch.setattr(pipeline.E, name, call)
    return r


def made(max_new=6, max_nodes=4, masses=True, fan_out=(2, 1)):
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations, EvictionPass
    ep = EvictionPass(P.Shape(2, 4, 2, 64, 4, [0, 40, 100]), [20, 30], device="cpu", dtype=torch.float32)
    return Continuations(ep, list(fan_out), max_new, P.Rope(0), 4, max_nodes, masses)


def tokens(n):
    return [torch.zeros(2, n, h, 64) for h in (4, 2, 2)]


def i32(v):
    return torch.tensor(v, dtype=torch.int32)


def test_trees_are_padded():
    co = made()
    t = co.tree([[-1, 0, 0], [-1], []])
    assert t.nodes == 3 and t.masks.tolist() == [[1, 3, 5], [1, 0, 0], [0, 0, 0]]
    rows, depths = t.steps
    assert rows[0].tolist() == [0, 1, 2] and rows[1, 0] == 0 and bool((rows[1, 1:] < -100).all()) and bool((rows[2] < -100).all())
    assert depths.tolist() == [[0, 1, 1], [0, 0, 0], [0, 0, 0]] and t.conts.tolist() == [0, 0, 0, 1, 1, 1, 2, 2, 2]
    assert co.tree([-1, 0]).masks.tolist() == [[1, 3]] * 3


def test_trees_are_refused():
    co = made()
    for bad, what in (([-1] * 5, "max_nodes"), ([], "max_nodes"), ([[-1]] * 2, "2 trees"), ([[], [], []], "max_nodes")):
        with pytest.raises(ValueError, match=what):
            co.tree(bad)
    with pytest.raises(Exception, match="earlier node"):
        co.tree([1, -1])
    with pytest.raises(ValueError, match="max_nodes"):
        made(max_nodes=65)
    with pytest.raises(ValueError, match="max_nodes"):
        made(max_nodes=0).tree([-1])


def test_a_draft_and_its_commit(rec):
    co = made()
    t = co.tree([[-1, 0, 1], [-1, -1], [-1]])
    co._at += i32([[1], [1], [5]])
    co.length = 1
    O = co.draft(*tokens(9), t, stream="s")
    assert [c[0] for c in rec.calls] == ["append", "decode_tree"]
    a, d = rec.calls[0][1], rec.calls[1][1]
    assert a[5].tolist() == [[45, 46, 47], [45, 45, 45], [65, 65, 65]]      # positions
    assert a[7][0].tolist() == [1, 2, 3] and a[7][1, :2].tolist() == [1, 2] and a[7][2, 0] == 1 and int(a[7][1, 2]) < 0
    assert a[9].shape == O.shape == (2, 4, 9, 64) and a[10] == d[-1] == "s"
    assert d[9].tolist() == [1, 1, 1] and d[10] == 1 and torch.equal(d[11], t.masks)
    path = i32([[0, 1, 2], [1, 0, 0], [0, 0, 0]])
    co.commit(path, i32([2, 1, 0]), longest=3)
    name, c, _ = rec.calls[2]
    assert name == "commit" and c[2].tolist() == [1, 1, 1] and c[-1] == "s"
    assert co.rows.tolist() == [3, 2, 1] and co.tail_counts.tolist() == [4, 3, 2] and co.positions.tolist() == [47, 46, 65] and co.length == 3
    co.accumulate(0.9)
    name, m, k = rec.calls[3]
    assert name == "accumulate" and m[9].tolist() == [3, 2, 1] and m[10] == 3
    assert torch.equal(m[13], path) and m[14].tolist() == [2, 1, 0] and m[15] == 0.9 and k == {"stream": "s"}
    assert m[0].shape == (2, 4, 9, 64) and m[1].shape == (2, 4, 9)


def test_the_bound_of_lengths(rec):
    co = made(max_new=6, max_nodes=4)
    t = co.tree([-1] * 4)
    for want in (4, 8):
        co.draft(*tokens(12), t)
        co.commit(i32([[0, 0, 0, 0]] * 3), i32([1, 1, 1]))
        assert co.length == want
    with pytest.raises(ValueError, match="hold 6"):
        co.draft(*tokens(12), t)
    with pytest.raises(ValueError, match="hold 6"):
        co.step(*tokens(3))
    assert co.tails.table.shape[1] * 4 >= 6 + 4
    co.evict(5, 3, 1)
    assert co.length == 5 and rec.calls[-1][0] == "evict_tails"
    co.step(*tokens(3))


def test_steps_are_weighed_before_and_after_they_are_advanced(rec):
    for first in (True, False):
        co = made()
        co.step(*tokens(3))
        if first:
            co.accumulate()
            co.advance()
        else:
            co.advance()
            co.accumulate()
        m = next(c[1] for c in rec.calls if c[0] == "accumulate")
        assert m[9].tolist() == [1, 1, 1] and m[10] == 1 and m[13] is None and m[14] is None and m[0].shape == (2, 4, 3, 64)
        with pytest.raises(ValueError, match="once"):
            co.accumulate()
        rec.calls.clear()


def test_evictions(rec):
    co = made()
    co._at[:2] += 4
    co.length = 4
    co.evict(3, 2, 1, stream="s")
    name, a, k = rec.calls[0]
    assert name == "evict_tails" and a[3:7] == [4, 3, 2, 1] and k["stream"] == "s" and co.length == 3
    assert co.tail_counts.tolist() == (co.rows + 1).tolist()
    co.evict_kept(15, 10, 2)
    name, a, k = rec.calls[1]
    assert name == "evict" and a[5:9] == [30, 15, 10, 2] and co.max_count == 15
    co.step(*tokens(3))
    assert rec.calls[-1][1][7] == 15


def test_calls_out_of_order_are_refused(rec):
    co = made()
    t = co.tree([-1, 0])
    path, acc = i32([[0, 1]] * 3), i32([1] * 3)
    with pytest.raises(ValueError, match="goes with a draft"):
        co.commit(path, acc)
    with pytest.raises(ValueError, match="step or a commit"):
        co.accumulate()
    co.step(*tokens(3))
    for f in (co.evict, co.evict_kept):
        with pytest.raises(ValueError, match="step is not finished"):
            f(3, 2, 1)
    co.advance()
    co.draft(*tokens(6), t)
    with pytest.raises(ValueError, match="commit"):
        co.advance()
    with pytest.raises(ValueError, match="step or a commit"):
        co.accumulate()
    with pytest.raises(ValueError, match="draft is not finished"):
        co.evict(3, 2, 1)
    with pytest.raises(ValueError, match="path has shape"):
        co.commit(i32([[0, 1, 2]] * 3), acc)
    co.commit(path, acc)
    co.evict(3, 2, 1)
    with pytest.raises(ValueError, match="step or a commit"):
        co.accumulate()  # (its rows may have moved)
    for n in (3, 5, 12):
        with pytest.raises(ValueError, match="3 x 2 nodes"):
            co.draft(*tokens(n), t)
    with pytest.raises(ValueError, match="continuations"):
        made(fan_out=(1, 1)).draft(*tokens(6), t)
    bare = made(masses=False)
    bare.step(*tokens(3))
    for f in (bare.accumulate, lambda: bare.evict(3, 2, 1), lambda: bare.evict_kept(3, 2, 1)):
        with pytest.raises(ValueError, match="without masses"):
            f()


def test_workspaces_that_were_outgrown_are_kept(rec):
    # a captured graph goes on using the one it was captured with
    co = made()
    first = co.workspace
    co._need(first.numel(), None)
    assert co.workspace is first
    co._need(first.numel() + 1, None)
    assert co.workspace is not first and co._outgrown == [first]


def test_a_draft_has_the_workspace_it_needs(rec):
    # shorter tails may be split otherwise and need more than the longest
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations, EvictionPass
    ep = EvictionPass(P.Shape(1, 28, 4, 128, 4, [0, 9000]), [6553], device="cpu")
    co = Continuations(ep, [1], 20000, P.Rope(0), 64, 64)
    t = co.tree([-1] * 64)
    for length in (0, 296, 333, 5000, 19999):
        co.length = length
        co.draft(*(torch.zeros(1, 64, h, 128) for h in (28, 4, 4)), t)
        assert rec.calls[-1][0] == "decode_tree" and rec.calls[-1][1][10] == length
        assert rec.calls[-1][1][14].numel() >= P.ecokv_decode_tree_workspace_size(ep.shape, co.fan, co.max_count, length, 64)
