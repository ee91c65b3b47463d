"""Masses behind the tails after a step that was accumulated, not advanced and replaced:
they are 0 in whichever pages the table names, and a tail that has run past its table
touches nobody else's.  The library's calls are replaced by recorders, the tensors are
the CPU's."""
import pytest
import torch

from test_drafts_host import i32, made, rec, tokens  # noqa: F401  (rec: a fixture)


@pytest.mark.parametrize("rows", [[0, 0, 0], [3, 4, 5], [7, 12, 0], [11, 12, 13], [40, 2, 2 ** 31 - 1]])
@pytest.mark.parametrize("then", ["step", "draft"])
def test_masses_behind_the_tails(rec, rows, then):  # noqa: F811
    co = made(max_new=8, max_nodes=4)          # three pages of four rows each
    P = co.tails.K.shape[1]
    assert co.tails.table.shape == (3, 3) and P == 9
    table = i32([[5, 0, 7], [8, 3, -1], [2, P, 4]])
    co.tails.table.copy_(table)
    co.rows.copy_(i32(rows))
    co.step(*tokens(3))
    co.accumulate()
    before = torch.rand(co.tail_mass.shape) + 1
    co.tail_mass.copy_(before)
    if then == "step":
        co.step(*tokens(3))
    else:
        co.draft(*tokens(6), co.tree([-1, 0]))
    want = before.clone()
    for c in range(3):
        for r in range(rows[c], 12):
            page = int(table[c, r // 4])
            if 0 <= page < P:
                want[:, page, :, r % 4] = 0
    assert torch.equal(co.tail_mass, want)
    # once
    co.tail_mass.copy_(before)
    co.step(*tokens(3))
    assert torch.equal(co.tail_mass, before)
