"""Host-side checks of ecokv_tree_masks, ecokv_decode_tree, ecokv_commit,
ecokv_accumulate, ecokv_evict and ecokv_evict_tails: every bad call returns its
error code before any device work (no GPU needed; the device addresses here are
never dereferenced)."""
import ctypes
import random

import pytest

from test_generate_abi import BAD_TAILS, E, P, at, tails  # noqa: F401  (fixtures)

ODD = ctypes.c_void_p(264)


def fan(*v):
    return (ctypes.c_int32 * len(v))(*v)


@pytest.mark.parametrize("n", [1, 2, 7, 63, 64])
def test_tree_masks(P, n):
    rng = random.Random(n)
    for _ in range(20):
        parents = [rng.randint(-1, i - 1) for i in range(n)]
        masks, depths = P.ecokv_tree_masks(parents)
        for i in range(n):
            want, node, depth = 0, i, -1
            while node >= 0:
                want, node, depth = want | 1 << node, parents[node], depth + 1
            assert masks[i] % 2 ** 64 == want and -2 ** 63 <= masks[i] < 2 ** 63 and depths[i] == depth
    assert P.ecokv_tree_masks(range(-1, n - 1))[1] == list(range(n))


@pytest.mark.parametrize("parents", [[], [-1] * 65, [0], [-1, 1], [-1, 2, 0], [-2], [-1, -2], [2 ** 31 - 1]])
def test_tree_masks_refuses(P, parents):
    with pytest.raises(P.EcoKVError) as e:
        P.ecokv_tree_masks(parents)
    assert e.value.code == -1


def test_tree_masks_of_null(E):
    n = (ctypes.c_int32 * 2)(-1, 0)
    out = (ctypes.c_uint64 * 2)()
    assert E.lib.ecokv_tree_masks(2, None, out, None) == -1 and E.lib.ecokv_tree_masks(2, n, None, None) == -1
    assert E.lib.ecokv_tree_masks(2, n, out, None) == 0 and out[:] == [1, 3]


BAD_FANS = [fan(1, 2, 5), fan(0, 3, 2), fan(0, -1, 5), None, fan(0, 1, 2 ** 31 - 1), fan(0, 1, 2 ** 27)]


def test_decode_tree_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100, 250])
    f, g = E.lib.ecokv_decode_tree, E.lib.ecokv_decode_tree_workspace_size
    n = ctypes.c_size_t(0)
    size = lambda fn=fan(0, 2, 5), mc=100, mt=30, m=6, out=n: g(ctypes.byref(s.c), fn, mc, mt, m, ctypes.byref(out) if out is not None else None)  # noqa: E731
    assert size() == 0 and n.value > 0
    ws = n.value
    for bad in BAD_FANS:
        assert size(fn=bad) == -1
    for kw in (dict(mc=-1), dict(mt=-30), dict(mt=2 ** 31 - 60), dict(m=0), dict(m=65), dict(m=-1), dict(out=None)):
        assert size(**kw) == -1, kw

    def call(Q=at(0), Kc=at(1), Vc=at(2), dtype=0, shape=s, fn=fan(0, 2, 5), cnt=at(3), off=at(4), mc=100, t=tails(E), tc=at(5), mt=30, m=6, masks=at(6),
             O=at(7), lse=at(8), w=at(9), wb=ws):
        return f(Q, Kc, Vc, dtype, ctypes.byref(shape.c), fn, cnt, off, mc, ctypes.byref(t) if t is not None else None, tc, mt, m, masks, O, lse, w, wb, None)

    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    for bad in BAD_FANS:
        assert call(fn=bad) == -1
    for m in ("Q", "Kc", "Vc", "cnt", "off", "O", "tc", "masks", "t", "w"):
        assert call(**{m: None}) == -1, m
    for m in ("Q", "Kc", "Vc", "O", "w"):
        assert call(**{m: ODD}) == -1, m
    assert call(dtype=3) == -3
    assert call(shape=P.Shape(2, 8, 2, 32, 4, [0, 100, 250])) == -3
    for kw in (dict(mc=-1), dict(mt=-1), dict(m=0), dict(m=65), dict(mt=129)):  # (8 pages of 16)
        assert call(**kw) == -1, kw
    assert call(t=tails(E, num_conts=4)) == -1
    assert call(wb=ws // 8) == -2
    # outputs over inputs, over each other
    for kw in (dict(O=at(0)), dict(O=at(10)), dict(O=at(11)), dict(lse=at(0)), dict(w=at(10)), dict(w=at(0)), dict(O=at(9)), dict(lse=at(9)), dict(lse=at(7))):
        assert call(**kw) == -1, kw
        assert "overlap" in P.ecokv_last_error(), kw
    assert call(fn=fan(0, 0, 0), Q=None) == 0                  # nobody continues
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100, 250]), Q=None) == 0


def test_commit_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100])

    def call(dtype=0, shape=s, t=tails(E), tc=at(0), m=6, path=at(1), acc=at(2)):
        return E.lib.ecokv_commit(dtype, ctypes.byref(shape.c), ctypes.byref(t) if t is not None else None, tc, m, path, acc, None)

    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    for m in ("t", "tc", "path", "acc"):
        assert call(**{m: None}) == -1, m
    for m in (0, -1, 65):
        assert call(m=m) == -1
    assert call(t=tails(E, V=ctypes.c_void_p(at(10).value + 4096))) == -1 and "overlap" in P.ecokv_last_error()
    assert call(dtype=7) == -3 and call(shape=P.Shape(2, 8, 2, 80, 4, [0, 100])) == -3
    assert call(t=tails(E, num_conts=0)) == 0
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100]), tc=None) == 0


def test_accumulate_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100, 250])

    def call(Q=at(0), lse=at(1), Kc=at(2), dtype=0, shape=s, fn=fan(0, 2, 5), cnt=at(3), off=at(4), mc=100, t=tails(E), tc=at(5), mt=30, m=6, path=at(6),
             acc=at(7), decay=1.0, mass=at(13), tm=at(14), mo=at(15), to=at(16)):
        return E.lib.ecokv_accumulate(Q, lse, Kc, dtype, ctypes.byref(shape.c), fn, cnt, off, mc, ctypes.byref(t) if t is not None else None, tc, mt, m, path,
                                      acc, ctypes.c_float(decay), mass, tm, mo, to, None)

    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    for bad in BAD_FANS:
        assert call(fn=bad) == -1
    for m in ("Q", "lse", "Kc", "cnt", "off", "t", "tc", "path", "acc", "mass", "tm", "mo", "to"):
        assert call(**{m: None}) == -1, m
    for m in ("Q", "Kc"):
        assert call(**{m: ODD}) == -1, m
    for bad in (-0.5, float("nan"), float("inf"), -float("inf")):
        assert call(decay=bad) == -1
    for kw in (dict(mc=-1), dict(mt=-1), dict(m=0), dict(m=65), dict(mt=129), dict(t=tails(E, num_conts=4)), dict(path=None, acc=None)):
        assert call(**kw) == -1, kw
    assert call(to=ctypes.c_void_p(at(14).value + 64)) == -1 and "overlap" in P.ecokv_last_error()
    assert call(dtype=3) == -3 and call(shape=P.Shape(2, 8, 2, 32, 4, [0, 100, 250])) == -3
    none = dict(Q=None, lse=None, Kc=None, cnt=None, off=None, t=None, tc=None, mass=None, tm=None, mo=None, to=None)
    assert call(mc=0, mt=0, **none) == 0
    assert call(mc=0, fn=fan(0, 0, 0), **none) == 0
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100, 250]), **none) == 0


BAD_KEEPS = [dict(limit=0, keep=0), dict(keep=0), dict(keep=21), dict(recent=-1), dict(recent=16), dict(limit=-5), dict(rows=-1)]


def test_evict_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100, 250])
    n = ctypes.c_size_t(0)
    size = lambda groups=2, rows=100, keep=15, out=n: E.lib.ecokv_evict_workspace_size(  # noqa: E731
        ctypes.byref(s.c), groups, rows, keep, ctypes.byref(out) if out is not None else None)
    assert size() == 0 and n.value == 4 * 8 * (4 + 2 * 15)
    ws = n.value
    for kw in (dict(groups=-1), dict(rows=-1), dict(keep=0), dict(out=None)):
        assert size(**kw) == -1, kw

    def call(Kc=at(0), Vc=at(1), dtype=0, shape=s, cnt=at(2), off=at(3), rows=100, limit=20, keep=15, recent=4, m=at(4), mo=at(5), new=at(6), w=at(7), wb=ws):
        return E.lib.ecokv_evict(Kc, Vc, dtype, ctypes.byref(shape.c), cnt, off, rows, limit, keep, recent, m, mo, new, w, wb, None)

    for kw in BAD_KEEPS:
        assert call(**kw) == -1, kw
    for m in ("Kc", "Vc", "cnt", "off", "m", "mo", "new", "w"):
        assert call(**{m: None}) == -1, m
    for m in ("Kc", "Vc", "w"):
        assert call(**{m: ODD}) == -1, m
    assert call(dtype=3) == -3 and call(shape=P.Shape(2, 8, 2, 32, 4, [0, 100, 250])) == -3
    assert call(wb=ws - 4) == -2
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100, 250]), Kc=None) == 0


def test_evict_tails_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100])
    ws = 4 * 2 * 2 * 5 * (4 + 2 * 15)

    def call(dtype=0, shape=s, t=tails(E), tc=at(0), rows=100, limit=20, keep=15, recent=4, m=at(1), mo=at(2), new=at(3), w=at(4), wb=ws):
        return E.lib.ecokv_evict_tails(dtype, ctypes.byref(shape.c), ctypes.byref(t) if t is not None else None, tc, rows, limit, keep, recent, m, mo, new, w, wb,
                                       None)

    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    for kw in BAD_KEEPS:
        assert call(**kw) == -1, kw
    for m in ("t", "tc", "m", "mo", "new", "w"):
        assert call(**{m: None}) == -1, m
    assert call(w=ODD) == -1 and call(rows=129) == -1          # (8 pages of 16)
    assert call(t=tails(E, V=ctypes.c_void_p(at(10).value + 4096))) == -1 and call(mo=ctypes.c_void_p(at(1).value + 64)) == -1
    assert "overlap" in P.ecokv_last_error()
    assert call(dtype=3) == -3 and call(shape=P.Shape(2, 8, 2, 32, 4, [0, 100])) == -3
    assert call(wb=ws - 4) == -2
    assert call(t=tails(E, num_conts=0)) == 0
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100]), tc=None) == 0


def test_the_binding_refuses_host_tensors_and_wrong_shapes(P):
    import torch
    s = P.Shape(1, 4, 2, 64, 4, [0, 10])
    pool, i = torch.zeros(1, 3, 2, 16, 64), torch.zeros(2, dtype=torch.int32)
    t = P.Tails(pool, pool.clone(), torch.zeros(1, 2, dtype=torch.int32))
    Q, K, masks = torch.zeros(1, 4, 3, 64), torch.zeros(5, 64), torch.zeros(1, 3, dtype=torch.int64)
    m, tm = torch.zeros(5), torch.zeros(1, 3, 2, 16)
    for f in (lambda: P.ecokv_decode_tree(Q, K, K, s, [0, 1], i, i, 5, t, i, 3, masks, Q.clone()),
              lambda: P.ecokv_commit(s, t, i, masks.int(), i),
              lambda: P.ecokv_accumulate(Q[:, :, :1], m, K, s, [0, 1], i, i, 5, t, i, 3, m, tm),
              lambda: P.ecokv_evict(K, K.clone(), s, i, i, 5, 4, 3, 1, m),
              lambda: P.ecokv_evict_tails(s, t, i, 5, 4, 3, 1, tm)):
        with pytest.raises(ValueError, match="GPU tensor"):
            f()
    for f in (lambda: P.ecokv_commit(s, None, i, masks.int(), i), lambda: P.ecokv_evict_tails(s, None, i, 5, 4, 3, 1, tm)):
        with pytest.raises(ValueError, match="tails is required"):
            f()
    with pytest.raises(ValueError, match="one entry per prompt"):
        P.ecokv_decode_tree_workspace_size(s, [0, 1, 2], 5, 0, 1)
    with pytest.raises(ValueError):
        P.ecokv_decode_tree_workspace_size(s, [0, 1], 2 ** 32 + 5, 0, 1)
    with pytest.raises(ValueError):
        P.ecokv_tree_masks([2 ** 32 - 1])
