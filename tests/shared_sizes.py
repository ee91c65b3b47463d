"""Sizes at which ecokv_decode_shared takes its wide query tiles over long parts,
and sizes past one dimension of its grids: run on the GPU by
tests/test_gpu_shared_wide.py, their splits checked on the host by
tests/test_shared_plan_wide.py."""

TAIL = 70  # longest tail of the wide calls

# dtype, D, L, Hq, Hkv, kept rows of each prompt's largest unit, fan, waves along the query rows,
# rows that a wave adds up at most
WIDE = [
    ("bf16", 128, 28, 28, 4, [2500], [16], 4, 1280),
    ("bf16", 128, 28, 28, 4, [2333, 300], [16, 3], 4, 1184),
    ("bf16", 128, 14, 64, 8, [2000], [40], 4, 1024),
    ("bf16", 64, 28, 32, 8, [3000], [20], 4, 1504),
    ("bf16", 64, 14, 32, 8, [4000, 3100], [9, 20], 4, 2016),
    ("f32", 128, 16, 28, 4, [1100], [9], 4, 288),
    ("f32", 64, 32, 16, 4, [2000], [16], 4, 1008),
    ("bf16", 128, 28, 16, 4, [2500], [12], 2, 640),
    ("bf16", 64, 28, 16, 4, [4100], [12], 2, 1056),
    ("f32", 128, 32, 16, 4, [1500], [6], 2, 384),
    ("f32", 64, 40, 16, 4, [2500], [6], 2, 432),
]


def kept(case):
    """[L][Hkv][B] kept rows: every head its own number, as where the heads of a layer share a budget."""
    _, _, L, _, Hkv, counts, _, _, _ = case
    return [[[n if (l, h) == (0, 0) else 1 if (l, h) == (1, 0) else n - 37 * ((5 * h + 3 * l + s) % 41) * n // 4000
              for s, n in enumerate(counts)] for h in range(Hkv)] for l in range(L)]


# L, Hq, Hkv, D, number of prompts (each continued once) or continuations of one, max_count, max_tail
GRID_TAILS = (2, 64, 64, 128, 65_600, 0, 1)             # tails, and the merge of a row's few partials
GRID_PROMPTS = (260, 64, 64, 64, 64, 1, 0)              # prompts' blocks
GRID_MERGE = (260, 64, 64, 64, 64, 25 << 22, 0)         # the merge of many partials, 25 million blocks

# rows that a head of 4 keeps on average where they share a budget, the most that one may, and a wave's of them
SHARED_BUDGET = 1600
SHARED_BOUND = 4 * (SHARED_BUDGET - 4) + 4
SHARED_WAVE = 736
