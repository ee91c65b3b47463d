"""ecokv_evict where the bound of a unit's rows is past what a block holds keys of in
registers: long units, short ones under a long bound, and both in one call."""
import sys

import pytest
import torch

from cache_cases import Cache
from test_gpu_evict import check_unit, masses

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_06663_amd  # noqa: F401  (fails loudly if the library is not built)


LONG = [  # dtype, D, limit, keep, recent, counts [Hkv][prompts], bound (0: the largest count), masses
    ("bf16", 128, 6000, 5000, 8, [[9001, 8192, 8193], [26000, 0, 6001]], 0, "plain"),
    ("f32", 64, 9000, 9000, 0, [[20001, 9000], [9001, 1]], 0, "ties"),
    ("bf16", 64, 100, 100, 100, [[8193, 101], [100, 30]], 0, "odd"),
    ("bf16", 128, 700, 350, 349, [[701, 1400], [699, 2049], [8191, 1]], 30000, "old"),
    ("f32", 128, 2047, 2047, 7, [[2048, 5000]], 8193, "same"),
    ("bf16", 128, 12000, 11000, 500, [[16384, 16385, 12001]], 40000, "odd"),
    ("bf16", 64, 1, 1, 0, [[9000, 2]], 0, "ties"),
]


@pytest.mark.parametrize("case", LONG, ids=lambda c: f"{c[0]}-D{c[1]}-{c[2]}-{c[3]}-{c[4]}-{c[6]}-{c[7]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_long_kept(case, in_place):
    import paper_2609_06663_amd as P
    dtype, D, limit, keep, recent, counts, bound, kind = case
    print(f"[gpu-evict] long {case} {in_place}", file=sys.stderr, flush=True)
    H, B = len(counts), len(counts[0])
    t = Cache(13, dtype, 1, H, H, D, [counts], [1] * B, [1] * B)
    bound = bound or t.max_count
    assert bound > 8192
    mass = masses(kind, t.g, (t.Kc.shape[0],))
    K, V, m = t.Kc.clone(), t.Vc.clone(), mass.clone()
    out = mass if in_place else torch.full_like(mass, -7.0)
    before = t.counts.tolist()
    new = t.counts if in_place else torch.full_like(t.counts, -7)
    ws = torch.full((P.ecokv_evict_workspace_size(t.shape, B, bound, keep),), 0xFF, dtype=torch.uint8, device="cuda")
    P.ecokv_evict(t.Kc, t.Vc, t.shape, t.counts, t.offsets, bound, limit, keep, recent, mass, new, out, ws)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert new.tolist() == [keep if n > limit else n for n in before]
    for n, o in zip(before, t.offsets.tolist()):
        s = slice(o, o + n)
        check_unit(K[s], V[s], m[s], t.Kc[s], t.Vc[s], out[s], n, limit, keep, recent, bits, in_place)


def test_the_bound_does_not_change_what_stays():
    """The same units under bounds of every form of the plan: the same bits."""
    import paper_2609_06663_amd as P
    t = Cache(14, "bf16", 2, 2, 2, 64, [[[2048, 900, 1025], [300, 2047, 0]], [[1, 64, 2000], [1999, 1500, 1024]]], [1] * 3, [1] * 3)
    mass = masses("ties", t.g, (t.Kc.shape[0],))
    got = []
    for bound in (2048, 2049, 8192, 8193, 50000):
        print(f"[gpu-evict] bound {bound}", file=sys.stderr, flush=True)
        K, V, m, n = t.Kc.clone(), t.Vc.clone(), mass.clone(), t.counts.clone()
        P.ecokv_evict(K, V, t.shape, n, t.offsets, bound, 1024, 1000, 33, m)
        torch.cuda.synchronize()
        got.append((K.view(torch.int16), V.view(torch.int16), m, n))
    for other in got[1:]:
        for x, y in zip(got[0][2:], other[2:]):
            assert torch.equal(x, y)
        for o, n in zip(t.offsets.tolist(), got[0][3].tolist()):
            assert torch.equal(got[0][0][o:o + n], other[0][o:o + n]) and torch.equal(got[0][1][o:o + n], other[1][o:o + n])
