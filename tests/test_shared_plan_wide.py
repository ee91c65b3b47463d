"""How ecokv_decode_shared splits the calls of tests/test_gpu_shared_wide.py:
their blocks have as many query rows as they are there for, and their parts
enough tiles to go round the stages many times, odd and even numbers of them;
and the other calls go past one dimension of each grid."""
import numpy as np
import pytest
from shared_sizes import GRID_MERGE, GRID_PROMPTS, GRID_TAILS, SHARED_BOUND, SHARED_BUDGET, SHARED_WAVE, TAIL, WIDE, kept
from test_shared_plan import lib  # noqa: F401  (a fixture)

GRID_X = 1 << 20


def ceil(a, b):
    return -(-a // b)


def plan(lib, L, Hq, Hkv, D, fan, max_count, max_tail, bf16):  # noqa: F811
    """np, nt, prompt blocks, tail waves, bytes, wq."""
    out = np.zeros(6, np.int64)
    cum = np.concatenate([[0], np.cumsum(fan)]).astype(np.int32)
    n = np.array([0, 1, max(max_count, max_tail)], np.int32)
    assert lib.plan(L * Hkv, Hq // Hkv, D, len(fan), cum.ctypes.data, max_count, max_tail, int(bf16), n.ctypes.data, len(n), out.ctypes.data) == 0
    return out.tolist()


@pytest.mark.parametrize("case", WIDE, ids=str)
def test_wide_tiles_over_long_parts(lib, case):  # noqa: F811
    dtype, D, L, Hq, Hkv, counts, fan, want, wave = case
    rows = 32 if dtype == "bf16" else 16
    np_, nt, _, _, _, wq = plan(lib, L, Hq, Hkv, D, fan, max(counts), TAIL, dtype == "bf16")
    assert wq == want and nt == 1
    groups = 4 // wq
    step = rows * groups
    tiles = set()
    for n in {n for layer in kept(case) for head in layer for n in head}:
        part = ceil(ceil(n, np_), step) * step
        for first in range(0, n, part):
            tiles.add(ceil(ceil(min(part, n - first), groups), rows))
    assert ceil(ceil(ceil(max(counts), np_), step) * step, groups) == wave
    assert max(tiles) >= 16 and {t % 2 for t in tiles if t >= 8} == {0, 1} and min(tiles) == 1, sorted(tiles)


def test_a_shared_budget_is_a_wide_call(lib):  # noqa: F811
    # 7 layers of 28 / 4 heads, 16 continuations: by the bound, not by the rows
    np_, _, _, _, _, wq = plan(lib, 7, 28, 4, 128, [16], SHARED_BOUND, 3, True)
    assert wq == 4 and ceil(ceil(SHARED_BOUND, np_), 32) * 32 == SHARED_WAVE
    assert plan(lib, 7, 28, 4, 128, [16], SHARED_BUDGET, 3, True)[5] == 1


def test_grids_past_one_dimension(lib):  # noqa: F811
    L, Hq, Hkv, D, N, mc, mt = GRID_TAILS
    np_, nt, _, waves, _, _ = plan(lib, L, Hq, Hkv, D, [N], mc, mt, True)
    assert (np_, nt) == (0, 1) and waves // 4 > GRID_X
    assert L * Hq * N // (256 // (D // 4)) > GRID_X                  # the merge: 256 threads, D / 4 for a row
    L, Hq, Hkv, D, B, mc, mt = GRID_PROMPTS
    np_, nt, blocks, _, _, _ = plan(lib, L, Hq, Hkv, D, [1] * B, mc, mt, True)
    assert (np_, nt) == (1, 0) and blocks > GRID_X
    L, Hq, Hkv, D, B, mc, mt = GRID_MERGE
    np_, nt, blocks, _, nbytes, _ = plan(lib, L, Hq, Hkv, D, [1] * B, mc, mt, True)
    assert np_ > 24 and L * Hq * B > GRID_X and blocks > 24 * GRID_X  # a block for a row
    assert nbytes < 8 << 30
