"""Host-side checks of ecokv_commit_taken: what ecokv_commit refuses, and where the
numbers of rows would go (no GPU needed; the device addresses are never dereferenced)."""
import ctypes

from test_generate_abi import BAD_TAILS, E, P, at, tails  # noqa: F401  (fixtures)


def test_commit_taken_refusals(P, E):  # noqa: F811
    s = P.Shape(2, 8, 2, 128, 4, [0, 100])

    def call(dtype=0, shape=s, t=tails(E), tc=at(0), m=6, path=at(1), acc=at(2), taken=at(3)):
        return E.lib.ecokv_commit_taken(dtype, ctypes.byref(shape.c), ctypes.byref(t) if t is not None else None, tc, m, path, acc, taken, None)

    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    for m in ("t", "tc", "path", "acc", "taken"):
        assert call(**{m: None}) == -1, m
    for m in (0, -1, 65):
        assert call(m=m) == -1
    for i in (0, 1, 2, 10, 11):
        assert call(taken=at(i)) == -1 and "overlap" in P.ecokv_last_error(), i
    assert call(dtype=7) == -3 and call(shape=P.Shape(2, 8, 2, 80, 4, [0, 100])) == -3
    assert call(t=tails(E, num_conts=0)) == 0
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100]), tc=None) == 0
