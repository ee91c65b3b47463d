"""Several Continuations with masses on one pass: an eviction of the pass's rows leaves
the others' masses in the old order, so they are not used.  The library's calls are
replaced by recorders, the tensors are the CPU's."""
import pytest
import torch

from test_drafts_host import made, rec, tokens  # noqa: F401  (rec: a fixture)


def two(rec, masses=True):  # noqa: F811
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    a = made()
    return a, Continuations(a.ep, [1, 1], 6, P.Rope(0), 4, 4, masses)


def test_masses_of_another_order_are_refused(rec):  # noqa: F811
    a, b = two(rec)
    b.step(*tokens(2))
    b.accumulate()
    b.advance()
    a.evict_kept(15, 10, 2)
    n = len(rec.calls)
    with pytest.raises(ValueError, match="another.*moved"):
        b.evict_kept(15, 10, 2)
    b.step(*tokens(2))
    with pytest.raises(ValueError, match="another.*moved"):
        b.accumulate()
    assert [c[0] for c in rec.calls[n:]] == ["append", "decode_shared"]
    b.advance()
    b.evict(5, 3, 1)               # (its own rows)
    # the one that evicted goes on, again and again
    a.step(*tokens(3))
    a.accumulate()
    a.advance()
    a.evict_kept(12, 8, 2)
    a.step(*tokens(3))
    a.accumulate()


def test_those_without_masses_go_on(rec):  # noqa: F811
    a, b = two(rec, False)
    a.evict_kept(15, 10, 2)
    b.step(*tokens(2))
    assert rec.calls[-1][0] == "decode_shared"


def test_one_that_is_made_later_begins_anew(rec):  # noqa: F811
    a, _ = two(rec)
    a.evict_kept(15, 10, 2)
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations
    c = Continuations(a.ep, [1, 1], 6, P.Rope(0), 4, 4, True)
    c.step(*tokens(2))
    c.accumulate()
    c.advance()
    assert not torch.any(c.mass)
    c.evict_kept(12, 8, 2)
    a.step(*tokens(3))
    with pytest.raises(ValueError, match="another.*moved"):
        a.accumulate()
