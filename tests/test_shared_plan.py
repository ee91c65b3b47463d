"""The arithmetic of ecokv_shared_plan.h, compiled here for the host: where a
paged row lies (pages outside the pool, rows and continuations outside the
table are found before anything is read), and how a call's rows are split:
every row of every unit and tail is in exactly one part, and every part has a
place in the workspace."""
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
#include "ecokv_shared_plan.h"
using namespace ecokv;
extern "C" int page_of(const int *table, int conts, int pages, int shift, int max_pages, int cont, int row) {
    return tail_page(TailMap{table, conts, pages, shift, max_pages}, cont, row);
}
extern "C" long long row_of(int pages, int shift, int Hkv, int l, int h, int page, int row) {
    return tail_row(TailMap{nullptr, 1, pages, shift, 1}, Hkv, l, h, page, row);
}
// a count of n rows: its parts hold its rows once, each a whole number of steps but the last
static int covers(int n, int parts, int step) {
    long long got = 0;
    const int used = parts_used(n, parts, step);
    if (used > parts) return 1;
    if (n <= 0) return used != 0;
    const long long pr = part_rows(n, parts, step);
    if (pr % step || pr > kShMostRows + 2 * step || (step & (step - 1))) return 2;
    for (int p = 0; p < parts; ++p) {
        const long long left = (long long)n - p * pr;
        if ((left > 0) != (p < used)) return 3;
        got += left < 0 ? 0 : left < pr ? left : pr;
    }
    return got == n ? 0 : 4;
}
extern "C" int plan(long long pairs, int G, int D, int B, const int *fan, int max_count, int max_tail, int bf16, const int *n, int nn, long long *out) {
    const SharedGrid g = shared_grid(pairs, G, D, B, fan, max_count, max_tail, bf16 != 0);
    out[0] = g.np, out[1] = g.nt, out[2] = g.prompt_blocks, out[3] = g.tail_waves, out[4] = (long long)g.bytes, out[5] = g.wq;
    const int N = fan[B], qt = g.wq * g.rows_q;
    if ((max_count > 0 && N > 0) != (g.np > 0) || g.prompt_blocks != pairs * g.tiles * g.np) return 10;
    if ((max_tail > 0 && N > 0) != (g.nt > 0) || g.tail_waves != pairs * N * g.groups * g.nt || g.groups * kTailQ < G) return 11;
    if (g.step != g.rows_t * (kShWaves / g.wq) || kShWaves % g.wq) return 14;
    for (int s = 0; s < B; ++s) {  // every query row of a prompt has one tile
        const long long M = (long long)G * (fan[s + 1] - fan[s]), t = g.tile0[s + 1] - g.tile0[s];
        if (t * qt < M || (M > 0 ? (t - 1) * qt >= M : t != 0)) return 12;
    }
    for (int i = 0; i < nn; ++i) {
        if (g.np > 0)
            if (int rc = covers(n[i] < max_count ? n[i] : max_count, g.np, g.step)) return rc;
        if (g.nt > 0)
            if (int rc = covers(n[i] < max_tail ? n[i] : max_tail, g.nt, g.tail_step)) return 20 + rc;
    }
    return g.bytes == 4ull * (g.np + g.nt) * pairs * G * N * (D + 2) ? 0 : 13;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared_plan")
    (d / "plan.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-fsanitize=undefined",
                           "-fno-sanitize-recover=undefined", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o",
                           str(d / "plan.so"), str(d / "plan.cpp")])
    lib = ctypes.CDLL(str(d / "plan.so"))
    lib.page_of.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 6
    lib.row_of.argtypes = [ctypes.c_int] * 7
    lib.row_of.restype = ctypes.c_longlong
    lib.plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                         ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    return lib


@pytest.mark.parametrize("shift", [0, 3, 6])
def test_pages_outside_the_pool_are_found(lib, shift):
    # the table lies between words that no call may read as its own
    conts, max_pages, pages = 3, 4, 7
    words = np.full(conts * max_pages + 16, 5, np.int32)
    table = words[8:-8].reshape(conts, max_pages)
    table[:] = [[0, 6, 7, -1], [-2 ** 31, 2 ** 31 - 1, 3, 1], [2, 100, -7, 6]]
    top = max_pages << shift
    for c in range(-2, conts + 3):
        for row in [-2 ** 31, -1, *range(0, top), top, top + 1, 2 ** 31 - 1]:
            want = -1
            if 0 <= c < conts and 0 <= row < top:
                p = int(table[c, row >> shift])
                want = p if 0 <= p < pages else -1
            assert lib.page_of(table.ctypes.data, conts, pages, shift, max_pages, c, row) == want, (c, row)


def test_rows_of_a_pool_past_32_bits(lib):
    # [L][pages][Hkv][page_size]
    for pages, shift, Hkv, l, h, page, row in [(7, 4, 3, 0, 0, 0, 0), (7, 4, 3, 1, 2, 6, 37), (2 ** 20, 16, 64, 27, 63, 2 ** 20 - 1, 2 ** 31 - 1),
                                               (5, 0, 2, 3, 1, 4, 9)]:
        want = (((l * pages + page) * Hkv + h) << shift) + row % (1 << shift)
        assert lib.row_of(pages, shift, Hkv, l, h, page, row) == want


@pytest.mark.parametrize("G", [1, 2, 4, 7, 8, 16, 17, 64])
def test_parts_cover_every_row_once(lib, G):
    rng = np.random.default_rng(G)
    out = np.zeros(6, np.int64)
    for pairs in (1, 2, 4, 32, 112, 900):
        for fan in ([1], [2], [8], [0, 3], [5, 1, 12, 0, 3], [64], [300], [0, 0], [1] * 64):
            cum = np.concatenate([[0], np.cumsum(fan)]).astype(np.int32)
            for mc, mt in ((0, 5), (1, 0), (128, 1), (129, 1024), (6553, 200), (65536, 777), (2 ** 31 - 1, 2 ** 31 - 1), (8191, 0)):
                top = max(mc, mt, 1)
                n = np.unique(np.clip(np.concatenate([[0, 1, 31, 32, 33, 127, 128, 129, mc, mt, top - 1, -5],
                                                      rng.integers(0, top, 20)]), -5, top)).astype(np.int32)
                for bf16 in (0, 1):
                    rc = lib.plan(pairs, G, 128, len(fan), cum.ctypes.data, mc, mt, bf16, n.ctypes.data, len(n), out.ctypes.data)
                    assert rc == 0, (rc, pairs, G, fan, mc, mt, bf16, out.tolist())
                    # one round of the device, or a few parts each (and those that 32-bit offsets reach)
                    assert out[2] <= 256 or out[0] <= max(8, -(-mc // 2 ** 22))
                    assert out[3] <= 2048 or out[1] == max(1, -(-mt // 2 ** 22))
