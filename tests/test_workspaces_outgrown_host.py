"""What Continuations keeps of workspaces that were outgrown (a captured graph may go on
using them): together less than the one in use, however often the bounds change.  The
library's calls are replaced by recorders, the tensors are the CPU's."""
import pytest
import torch

from test_drafts_host import rec  # noqa: F401  (a fixture)


@pytest.mark.parametrize("L,Hq,Hkv,D,kept,fan_out,max_new,nodes", [
    (1, 4, 2, 64, [5659], [5], 11240, 31),
    (1, 2, 2, 128, [900, 6662], [0, 1], 12903, 46),
    (4, 1, 1, 64, [81, 70, 60], [0, 3, 1], 4325, 29),
    (1, 28, 4, 128, [6553], [1], 20000, 64),
])
def test_outgrown_workspaces_are_bounded(rec, L, Hq, Hkv, D, kept, fan_out, max_new, nodes):  # noqa: F811
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations, EvictionPass
    ep = EvictionPass(P.Shape(L, Hq, Hkv, D, 4, [9000 * i for i in range(len(kept) + 1)]), kept, device="cpu")
    co = Continuations(ep, fan_out, max_new, P.Rope(0), 64, nodes)
    most = 0
    for m in (nodes, nodes // 2):
        for length in range(0, max_new + 1, max_new // 200):
            need = P.ecokv_decode_tree_workspace_size(ep.shape, co.fan, co.max_count, length, m)
            co._need(need, None)
            assert co.workspace.numel() >= need
            most = max(most, need)
    assert all(isinstance(w, torch.Tensor) for w in co._outgrown)
    assert sum(w.numel() for w in co._outgrown) < co.workspace.numel() <= max(2 * most, P.ecokv_decode_tree_workspace_size(
        ep.shape, co.fan, co.max_count, max_new, nodes))
