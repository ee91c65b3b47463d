"""ecokv_decode_tree on bf16 rows: how exactly a weight meets the values.

Few rows with logits near each other, so that every weight is a large part of O, and
many values of O near 0, whose own rounding hides nothing.

Tolerance.  dx bounds a logit's error (cache_cases.logit_error); weights, their sums
and merges are off by at most 2 dx + 2^-18 of themselves, as in test_gpu_tree.py.  A
weight is the sum of two bf16 numbers, each cut and leaving less than a step, 2^-7, of
what it is cut from: 2^-14 of the weight.  O is rounded once, half a step of 2^-8:
  e = (2 dx + 2^-18) max |V| + 2^-14 sum_j w_j |v_j|,  |O - O64| <= e + 2^-8 (|O64| + e).
"""
import sys

import pytest
import torch

from cache_cases import logit_error
from test_gpu_tree import Trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


def check(t, O):
    _, Hq, Hkv, D, _ = t.dims
    G, M = Hq // Hkv, t.nodes
    small = 0
    for l in range(t.dims[0]):
        for h in range(Hkv):
            for c in range(t.N):
                x, K, V, seen, q = t.reference(l, h, c)
                rows = seen.any(0)
                K, V = torch.where(rows[:, None], K, 0.0), torch.where(rows[:, None], V, 0.0)
                live = seen.any(1)
                w = x[live].softmax(-1)
                ref = w @ V
                got = O[l, h * G:(h + 1) * G, c * M:(c + 1) * M].double().transpose(0, 1)[live]
                e = (2 * logit_error(q.reshape(M * G, D), K, D) + 2.0 ** -18) * float(V.abs().max()) + 2.0 ** -14 * (w @ V.abs())
                off = (got - ref).abs() - e - 2.0 ** -8 * (ref.abs() + e)
                assert bool((off <= 0).all()), (l, h, c, float(off.max()), int((off > 0).sum()))
                small += int((ref.abs() < 0.05).sum())
    assert small > 100


@pytest.mark.parametrize("D,Hq,Hkv,counts,fan,tails,nodes,bound", [
    (128, 28, 4, [9], [2], [0, 0], 5, 9),                      # kept rows, tiles of a wave
    (64, 8, 8, [7], [3], [0, 1, 0], 12, 7),
    (128, 28, 4, [9, 6], [4, 3], [0] * 7, 13, 3_000_000),      # tiles of a block
    (64, 16, 4, [8], [5], [0] * 5, 30, 3_000_000),
    (128, 8, 2, [0], [3], [6, 9, 11], 3, 0),                   # tails, by four waves
    (128, 4, 4, [0], [2], [40, 7], 60, 0),
    (64, 8, 2, [0], [3], [6, 9, 11], 5, 0),                    # tails, by one
    (64, 4, 4, [0], [2], [6, 9], 60, 0),
])
def test_weights_of_bf16_rows(D, Hq, Hkv, counts, fan, tails, nodes, bound):
    print(f"[gpu-tree] weights: {D} {Hq}/{Hkv} {counts} {fan} {tails} {nodes} nodes, bound {bound}", file=sys.stderr, flush=True)
    t = Trees(31, "bf16", 1, Hq, Hkv, D, [[counts] * Hkv], fan, tails, nodes, page=8, kscale=0.25)
    check(t, t.run(max_count=bound)[0])
