"""The arithmetic of ecokv_tree_plan.h and ecokv_evict_plan.h, compiled here for the
host: every kept row, every row of a tail and every drafted row is in exactly one
part, every part has a place in the workspace, and an eviction's plan has room for
every row that may move."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_06663_amd", "csrc")

SHIM = r"""
#define __host__
#define __device__
#include "ecokv_tree_plan.h"
#include "ecokv_evict_plan.h"
using namespace ecokv;
static int covers(int n, int parts, int step) {
    long long got = 0;
    const int used = parts_used(n, parts, step);
    if (used > parts) return 1;
    if (n <= 0) return used != 0;
    const long long pr = part_rows(n, parts, step);
    if (pr % step || pr > kShMostRows + 2 * step || (step & (step - 1))) return 2;
    for (int p = 0; p < used; ++p) {
        const long long left = (long long)n - p * pr;
        if (left <= 0) return 3;
        got += left < pr ? left : pr;
    }
    return got == n ? 0 : 4;
}
extern "C" int tree(long long pairs, int G, int D, int B, const int *fan, int conts, int nodes, int max_count, int max_tail, int bf16, const int *n,
                    int nn, long long *out) {
    TreeTails t{};
    TreeEven even{};
    const SharedGrid g = tree_grid(pairs, G, D, B, fan, conts, nodes, max_count, max_tail, bf16 != 0, &t, &even);
    out[0] = g.np, out[1] = g.nt, out[2] = g.prompt_blocks, out[3] = t.blocks, out[4] = (long long)g.bytes, out[5] = t.rows;
    out[6] = even.least, out[7] = even.fill, out[8] = 2 * g.rows_t;
    for (int s = 0; s <= B; ++s) out[9 + s] = g.tile0[s];
    const int qt = g.wq * g.rows_q, tt = t.wq * g.rows_q;
    if ((g.wq != 1 && g.wq != 4) || (t.wq != 1 && t.wq != 4)) return 10;
    if ((max_count > 0) != (g.np > 0) || g.prompt_blocks != (even.fill ? even.fill + pairs * g.tiles : pairs * g.tiles * g.np) || g.step != g.rows_t * (kShWaves / g.wq)) return 11;
    for (int s = 0; s < B; ++s) {
        const long long M = (long long)G * (fan[s + 1] - fan[s]), k = g.tile0[s + 1] - g.tile0[s];
        if (k * qt < M || (M > 0 ? (k - 1) * qt >= M : k != 0)) return 12;
    }
    // tails: tiles hold the query rows, parts the rows
    if ((long long)t.tiles * tt < (long long)nodes * G || (long long)(t.tiles - 1) * tt >= (long long)nodes * G) return 13;
    const long long rows = (long long)max_tail + nodes;
    if (g.nt < 1 || t.rows < 1 || t.rows % g.tail_step || (long long)g.nt * t.rows < rows) return 14;
    const long long items = pairs * conts * t.tiles * g.nt;
    if (t.wq == 1 ? g.tail_waves != items || t.blocks != (items + kShWaves - 1) / kShWaves : t.blocks != items) return 15;
    if (even.fill && (g.wq != 4 || even.least > g.np || even.fill < pairs * g.tiles * even.least || pairs * B > kEvenUnits)) return 17;
    for (int i = 0; i < nn; ++i)
        if (g.np > 0)
            if (int rc = covers(n[i] < max_count ? n[i] : max_count, g.np, g.step)) return rc;
    return g.bytes == 4ull * (g.np + g.nt) * pairs * G * fan[B] * (D + 2) + (even.fill ? kEvenBytes : 0) ? 0 : 16;
}
extern "C" int mass(long long pairs, int B, int conts, int max_count, int max_tail, long long *out) {
    int kp, tp;
    int64_t kb, tb;
    mass_grid(pairs, B, conts, max_count, max_tail, &kp, &tp, &kb, &tb);
    out[0] = kp, out[1] = tp, out[2] = kb, out[3] = tb;
    const long long each = kMassRows * kMassWaves;
    if ((max_count > 0) != (kp > 0) || kb != pairs * B * kp || (max_tail > 0 && conts > 0) != (tp > 0) || tb != pairs * conts * tp) return 1;
    // no block without a piece, none with more than eight
    if (kp > 0 && ((kp - 1) * each >= max_count || kp * each * 8 < max_count)) return 2;
    return tp > 0 && ((tp - 1) * each >= max_tail || tp * each * 8 < max_tail) ? 3 : 0;
}
extern "C" long long words(int max_rows, int keep) { return evict_plan_words(max_rows, keep); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_plan")
    (d / "plan.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-fsanitize=undefined",
                           "-fno-sanitize-recover=undefined", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o",
                           str(d / "plan.so"), str(d / "plan.cpp")])
    lib = ctypes.CDLL(str(d / "plan.so"))
    i, ll, p = ctypes.c_int, ctypes.c_longlong, ctypes.c_void_p
    lib.tree.argtypes = [ll, i, i, i, p, i, i, i, i, i, p, i, p]
    lib.mass.argtypes = [ll, i, i, i, i, p]
    lib.words.argtypes, lib.words.restype = [i, i], ll
    return lib


def cover_by_counts(rng, out, pairs, B, max_count, kind):
    """Parts by the counts: as the kernel works them out, every row of every tile is some block's, none past the grid or the workspace's places."""
    parts, blocks, least, fill, step = (int(out[i]) for i in (0, 2, 6, 7, 8))
    tiles = np.tile(np.diff(out[9:10 + B]), pairs).astype(np.int64)
    n = [np.full(pairs * B, max_count), rng.integers(0, max_count + 1, pairs * B), np.zeros(pairs * B),
         np.where(rng.random(pairs * B) < 0.1, max_count, 1)][kind].astype(np.int64)
    steps = -(-n // step)
    most = int((steps * (tiles > 0)).max())
    want = int(np.ceil(np.float32((tiles * steps).sum()) / np.float32(fill)))
    each = max(min(max(want, -(-most // parts)), -(-most // least)), 1)
    used = -(-steps // each)
    assert int((tiles * used).sum()) <= blocks and int((used * (tiles > 0)).max(initial=0)) <= parts
    assert bool((used * each >= steps).all()) and bool(((used - 1) * each < np.maximum(steps, 1)).all())


@pytest.mark.parametrize("G", [1, 2, 4, 7, 16, 64])
@pytest.mark.parametrize("nodes", [1, 5, 16, 64])
def test_tree_parts_cover_every_row_once(lib, G, nodes):
    rng = np.random.default_rng(G)
    out = np.zeros(9 + 65, np.int64)
    for pairs in (1, 4, 32, 112, 900):
        for fan in ([1], [8], [0, 3], [5, 1, 12, 0, 3], [64], [1] * 64):
            conts = np.concatenate([[0], np.cumsum(fan)])
            cum = (nodes * conts).astype(np.int32)
            for mc, mt in ((0, 5), (0, 0), (1, 0), (128, 1), (129, 1024), (6553, 200), (65536, 777), (2 ** 31 - 1, 2 ** 31 - 65), (8191, 0)):
                n = np.unique(np.clip(np.concatenate([[0, 1, 31, 32, 33, 127, 128, 129, mc, mc - 1, -5], rng.integers(0, max(mc, 1), 20)]),
                                      -5, max(mc, 1))).astype(np.int32)
                for bf16 in (0, 1):
                    for D in (64, 128):
                        rc = lib.tree(pairs, G, D, len(fan), cum.ctypes.data, int(conts[-1]), nodes, mc, mt, bf16, n.ctypes.data, len(n), out.ctypes.data)
                        assert rc == 0, (rc, pairs, fan, mc, mt, bf16, D, out.tolist())
                        if out[7] and (D == 128) == bool(bf16):
                            for kind in range(4):
                                cover_by_counts(rng, out, pairs, len(fan), mc, kind)


def test_pieces_of_masses(lib):
    out = np.zeros(4, np.int64)
    for pairs in (1, 4, 112, 2000):
        for B, conts in ((1, 1), (3, 70), (1, 0), (64, 64)):
            for mc in (0, 1, 127, 128, 129, 6553, 2 ** 31 - 1):
                for mt in (0, 1, 200, 5000, 2 ** 31 - 65):
                    rc = lib.mass(pairs, B, conts, mc, mt, out.ctypes.data)
                    assert rc == 0, (rc, pairs, B, conts, mc, mt, out.tolist())


def test_plans_hold_what_may_move(lib):
    for rows in (0, 1, 5, 100, 2 ** 31 - 1):
        for keep in (1, 2, 50, 99, 100, 101, 2 ** 30, 2 ** 31 - 1):
            # of n rows with n - keep that go, as many move as are dropped below `keep`
            most = max(0, min(keep, rows - keep))
            assert lib.words(rows, keep) == 4 + 2 * most
