"""What a step or a draft that the library refuses leaves behind: nothing that a later
accumulate or commit would take for the one before.  The library's calls are replaced by
recorders, the tensors are the CPU's."""
import pytest
import torch

from test_drafts_host import i32, made, rec, tokens  # noqa: F401  (rec: a fixture)


def refuse(monkeypatch, name):
    """Context: the library's call of this name raises."""
    from paper_2609_06663_amd import pipeline

    def call(*a, **k):
        raise ValueError(f"{name} refused")

    m = monkeypatch.context()
    with m as c:
        c.setattr(pipeline.E, name, call)
        yield


@pytest.fixture
def refused(monkeypatch):
    import contextlib
    return lambda name: contextlib.contextmanager(refuse)(monkeypatch, name)


def committed(co, nodes=2):
    t = co.tree([-1] * nodes)
    co.draft(*tokens(3 * nodes), t)
    path, acc = i32([list(range(nodes))] * 3), i32([1] * 3)
    co.commit(path, acc)
    return path


def test_a_draft_refused_before_anything_was_enqueued(rec, refused):  # noqa: F811
    # the commit before it can still be accumulated, with its own queries
    co = made()
    path = committed(co)
    Q = co.Q_nodes
    for name in ("ecokv_append", "ecokv_decode_tree_workspace_size"):
        with refused(name), pytest.raises(ValueError, match="refused"):
            co.draft(*tokens(12), co.tree([-1] * 4))
    assert co.Q_nodes is Q and co.lse_nodes.shape[2] == 6
    co.accumulate()
    assert rec.calls[-1][0] == "accumulate" and rec.calls[-1][1][0].shape[2] == 6 and torch.equal(rec.calls[-1][1][13], path)


def test_a_draft_refused_after_its_rows_were_appended(rec, refused):  # noqa: F811
    # its queries and rows took the place of the last draft's
    co = made()
    committed(co)
    with refused("ecokv_decode_tree"), pytest.raises(ValueError, match="refused"):
        co.draft(*tokens(12), co.tree([-1] * 4))
    with pytest.raises(ValueError, match="step or a commit"):
        co.accumulate()
    with pytest.raises(ValueError, match="goes with a draft"):
        co.commit(i32([[0, 1, 2, 3]] * 3), i32([1] * 3))
    co.evict(5, 3, 1)
    # nor is a draft that it replaced there any more
    co.draft(*tokens(6), co.tree([-1] * 2))
    with refused("ecokv_decode_tree"), pytest.raises(ValueError, match="refused"):
        co.draft(*tokens(12), co.tree([-1] * 4))
    for M in (2, 4):
        with pytest.raises(ValueError, match="goes with a draft"):
            co.commit(i32([list(range(M))] * 3), i32([1] * 3))


def test_a_draft_refused_for_its_shape_changes_nothing(rec):  # noqa: F811
    co = made()
    t = co.tree([-1, 0])
    co.draft(*tokens(6), t)
    with pytest.raises(ValueError, match="3 x 4 nodes"):
        co.draft(*tokens(6), co.tree([-1] * 4))
    co.commit(i32([[0, 1]] * 3), i32([2] * 3))
    co.accumulate()


@pytest.mark.parametrize("advanced", [False, True])
def test_a_step_refused(rec, refused, advanced):  # noqa: F811
    co = made()
    co.step(*tokens(3))
    if advanced:
        co.advance()
    with refused("ecokv_append"), pytest.raises(ValueError, match="refused"):
        co.step(*tokens(3))
    co.accumulate()  # (nothing was enqueued)
    assert rec.calls[-1][0] == "accumulate"
    co.step(*tokens(3))
    with refused("ecokv_decode_shared"), pytest.raises(ValueError, match="refused"):
        co.step(*tokens(3))
    with pytest.raises(ValueError, match="step or a commit"):
        co.accumulate()


def test_the_stream_of_a_refused_call_is_not_the_next_ones(rec, refused):  # noqa: F811
    co = made()
    co.step(*tokens(3), stream="s")
    with refused("ecokv_append"):
        with pytest.raises(ValueError, match="refused"):
            co.step(*tokens(3), stream="t")
        with pytest.raises(ValueError, match="refused"):
            co.draft(*tokens(6), co.tree([-1, 0]), stream="t")
    co.accumulate()
    assert rec.calls[-1][2]["stream"] == "s"
