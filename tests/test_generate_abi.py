"""Host-side checks of ecokv_rope_freqs, ecokv_prefill_rope, ecokv_append and
ecokv_decode_shared: every bad call returns its error code before any device
work (no GPU needed; the device addresses here are never dereferenced)."""
import ctypes
import math

import pytest


@pytest.fixture(scope="module")
def P():
    import paper_2609_06663_amd as P
    return P


@pytest.fixture(scope="module")
def E(P):
    from paper_2609_06663_amd import ecokv as E
    return E


def at(i):
    """A fake device address, 2^40 bytes from the next."""
    return ctypes.c_void_p((i + 1) << 40)


def want_freqs(rot, base, kind, stretch, context):
    out = []
    if kind == 2:
        base = base * stretch ** (rot / (rot - 2))
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if kind == 1:
            f /= stretch
        if kind == 3:
            turns = context * f / (2 * math.pi)
            keep = min(max((turns - 1) / 31, 0.0), 1.0)
            f = f * keep + f / stretch * (1 - keep)
        out.append(f)
    return out, 0.1 * math.log(stretch) + 1 if kind == 3 else 1.0


@pytest.mark.parametrize("rot", [2, 4, 16, 64, 96, 128])
@pytest.mark.parametrize("kind,stretch,context", [(0, 1.0, 0.0), (1, 8.0, 0.0), (2, 4.0, 0.0), (3, 16.0, 4096.0), (3, 1.0, 2048.0)])
def test_rope_freqs(P, rot, kind, stretch, context):
    if kind == 2 and rot == 2:
        with pytest.raises(P.EcoKVError):
            P.ecokv_rope_freqs(rot, 10000.0, kind, stretch)
        return
    got, factor = P.ecokv_rope_freqs(rot, 10000.0, kind, stretch, context)
    want, wf = want_freqs(rot, 10000.0, kind, stretch, context)
    # (rounded to float32 once, from a handful of double operations)
    assert len(got) == rot // 2 and all(abs(g - w) <= 2.0 ** -24 * w * 1.0001 for g, w in zip(got, want))
    assert abs(factor - wf) <= 2.0 ** -24 * wf


@pytest.mark.parametrize("args", [(0,), (3,), (-2,), (16, 1.0), (16, float("inf")), (16, float("nan")), (16, 1e4, 4), (16, 1e4, -1), (16, 1e4, 1, 0.5),
                                  (16, 1e4, 1, float("nan")), (16, 1e4, 3, 2.0, 0.0), (16, 1e4, 3, 2.0, float("inf")), (4, 1e300, 2, 1e300)])
def test_rope_freqs_rejects(P, args):
    with pytest.raises(P.EcoKVError) as e:
        P.ecokv_rope_freqs(*args)
    assert e.value.code == -1


def rope(E, **kw):
    f = dict(rot_dim=128, interleaved=0, freq=at(30), factor=1.0, norm_eps=1e-6, q_norm=None, k_norm=None)
    f.update(kw)
    return E._Rope(*(f[n] for n, _ in E._Rope._fields_))


BAD_ROPES = [(dict(rot_dim=-16), -1), (dict(rot_dim=130), -1), (dict(rot_dim=144), -1), (dict(rot_dim=17), -1), (dict(rot_dim=24), -3), (dict(rot_dim=2), -3),
             (dict(interleaved=2), -1), (dict(freq=None), -1), (dict(factor=float("nan")), -1), (dict(factor=float("inf")), -1),
             (dict(norm_eps=-1.0), -1), (dict(norm_eps=float("nan")), -1), (dict(q_norm=ctypes.c_void_p(264)), -1), (dict(k_norm=ctypes.c_void_p(264)), -1)]


def test_prefill_rope_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100, 110])
    f = E.lib.ecokv_prefill_rope

    def call(Q=at(0), qs=1024, K=at(1), ks=256, dtype=0, shape=s, rp=None, pos=at(2), Qo=at(3), Ko=at(4), win=at(5)):
        return f(Q, qs, K, ks, dtype, ctypes.byref(shape.c), ctypes.byref(rp or rope(E)), pos, Qo, Ko, win, None)

    for kw, code in BAD_ROPES:
        assert call(rp=rope(E, **kw)) == code, kw
    assert call(dtype=2) == -3
    assert call(shape=P.Shape(2, 8, 2, 96, 4, [0, 100])) == -3
    assert call(shape=P.Shape(2, 8, 3, 128, 4, [0, 100])) == -1
    assert call(shape=P.Shape(2, 8, 2, 128, 4, [0, 100, 100])) == -1       # an empty sequence
    assert call(shape=P.Shape(2, 8, 2, 128, 0, [0, 100])) == -1            # a window of 0 with Q_win
    assert call(shape=P.Shape(2, 8, 2, 128, 11, [0, 100, 110])) == -1      # longer than a sequence
    assert "window" in P.ecokv_last_error()
    assert call(K=None) == -1 and call(Ko=None) == -1                      # both or neither
    assert call(Q=None) == -1 and call(Qo=None, win=None) == -1
    assert call(qs=1023) == -1 and call(ks=252) == -1 and call(qs=1028) == -1 and call(qs=-1024) == -1
    for n in ("Q", "K", "Qo", "Ko", "win"):
        assert call(**{n: ctypes.c_void_p((1 << 45) + 8)}) == -1, n        # not 16-byte aligned
    assert call(Qo=at(0), qs=1032) == -1                                   # in place, not packed
    assert call(Qo=ctypes.c_void_p((1 << 40) + 2048)) == -1                # partly in place
    assert call(Ko=ctypes.c_void_p(at(1).value + 512)) == -1
    assert call(Qo=at(4)) == -1 and call(win=at(3)) == -1 and call(win=at(4)) == -1 and call(Ko=at(0)) == -1 and call(win=at(0)) == -1
    assert "overlap" in P.ecokv_last_error()
    assert call(qs=1 << 62) == -1
    assert call(shape=P.Shape(1, 1 << 24, 1, 128, 4, [0, 9]), qs=1 << 31, ks=128) == -1   # a token of 2^31 elements
    assert f(None, 0, None, 0, 0, ctypes.byref(P.Shape(0, 8, 2, 128, 4, [0, 9]).c), ctypes.byref(rope(E)), None, None, None, None, None) == 0
    assert f(None, 0, None, 0, 0, ctypes.byref(s.c), ctypes.byref(rope(E)), None, None, None, None, None) == 0   # nothing asked for
    assert f(None, 0, None, 0, 0, ctypes.byref(s.c), None, None, None, None, None, None) == -1


def tails(E, **kw):
    t = dict(K=at(10), V=at(11), table=at(12), num_conts=5, num_pages=40, page_size=16, max_pages=8)
    t.update(kw)
    return E._Tails(*(t[n] for n, _ in E._Tails._fields_))


BAD_TAILS = [dict(K=None), dict(V=None), dict(table=None), dict(num_conts=-1), dict(num_pages=0), dict(page_size=0), dict(page_size=24), dict(page_size=-16),
             dict(page_size=131072), dict(max_pages=0), dict(max_pages=1 << 28), dict(K=ctypes.c_void_p(264)), dict(V=ctypes.c_void_p(264))]


def test_append_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100])
    f = E.lib.ecokv_append

    def call(Q=at(0), qs=1024, K=at(1), ks=256, V=at(2), vs=256, dtype=0, shape=s, rp=None, pos=at(3), conts=None, rows=at(4), n=5, t=None, Qd=at(5)):
        return f(Q, qs, K, ks, V, vs, dtype, ctypes.byref(shape.c), ctypes.byref(rp or rope(E)), pos, conts, rows, n, ctypes.byref(t or tails(E)), Qd, None)

    for kw, code in BAD_ROPES:
        assert call(rp=rope(E, **kw)) == code, kw
    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    assert call(dtype=7) == -3 and call(n=-1) == -1
    assert call(shape=P.Shape(2, 8, 2, 80, 4, [0, 100])) == -3
    assert call(n=6) == -1                                     # more tokens than continuations, without conts
    for n in ("K", "V", "pos", "rows", "Q", "Qd"):
        assert call(**{n: None}) == -1, n
    for n in ("Q", "K", "V", "Qd"):
        assert call(**{n: ctypes.c_void_p((1 << 45) + 8)}) == -1, n
    assert call(qs=1020) == -1 and call(ks=128) == -1 and call(vs=260) == -1
    assert call(Qd=at(0)) == -1 and call(Qd=at(10)) == -1 and call(K=at(11)) == -1
    assert call(t=tails(E, V=ctypes.c_void_p(at(10).value + 4096))) == -1
    assert "overlap" in P.ecokv_last_error()
    assert call(n=0, K=None) == 0                              # nothing to do
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100]), K=None) == 0


def test_decode_shared_refusals(P, E):
    s = P.Shape(2, 8, 2, 128, 4, [0, 100, 250])
    f, g = E.lib.ecokv_decode_shared, E.lib.ecokv_decode_shared_workspace_size
    fan = lambda *v: (ctypes.c_int32 * len(v))(*v)
    n = ctypes.c_size_t(0)
    assert g(ctypes.byref(s.c), fan(0, 2, 5), 100, 30, ctypes.byref(n)) == 0 and n.value > 0
    ws = n.value
    for bad in (fan(1, 2, 5), fan(0, 3, 2), fan(0, -1, 5), None, fan(0, 1, 2 ** 31 - 1)):
        assert g(ctypes.byref(s.c), bad, 100, 30, ctypes.byref(n)) == -1
    assert g(ctypes.byref(s.c), fan(0, 2, 5), -1, 30, ctypes.byref(n)) == -1
    assert g(ctypes.byref(s.c), fan(0, 2, 5), 1, -30, ctypes.byref(n)) == -1
    assert g(ctypes.byref(s.c), fan(0, 2, 5), 1, 30, None) == -1

    def call(Q=at(0), Kc=at(1), Vc=at(2), dtype=0, shape=s, fn=fan(0, 2, 5), cnt=at(3), off=at(4), mc=100, t=None, tc=at(5), mt=30, O=at(6), w=at(7), wb=ws):
        return f(Q, Kc, Vc, dtype, ctypes.byref(shape.c), fn, cnt, off, mc, ctypes.byref(t) if t is not None else None, tc, mt, O, None, w, wb, None)

    good = tails(E)
    for kw in BAD_TAILS:
        assert call(t=tails(E, **kw)) == -1, kw
    assert call() == -1                                        # no tails
    assert call(t=good, fn=None) == -1 and call(t=good, fn=fan(0, 3, 2)) == -1
    for m in ("Q", "Kc", "Vc", "cnt", "off", "O", "tc"):
        assert call(t=good, **{m: None}) == -1, m
    for m in ("Q", "Kc", "Vc", "O"):
        assert call(t=good, **{m: ctypes.c_void_p(264)}) == -1, m
    assert call(t=good, dtype=3) == -3
    assert call(t=good, shape=P.Shape(2, 8, 2, 32, 4, [0, 100, 250])) == -3
    assert call(t=good, mc=-1) == -1 and call(t=good, mt=-1) == -1
    assert call(t=good, mt=129) == -1                          # more than 8 pages of 16
    assert call(t=tails(E, num_conts=4)) == -1
    assert call(t=good, w=None) == -1 and call(t=good, w=ctypes.c_void_p(260)) == -1
    assert call(t=good, wb=1024) == -2
    assert call(fn=fan(0, 0, 0), Q=None) == 0                  # nobody continues
    assert call(shape=P.Shape(0, 8, 2, 128, 4, [0, 100, 250]), Q=None) == 0


def test_the_binding_refuses_host_tensors_and_wrong_shapes(P):
    import torch
    s = P.Shape(1, 4, 2, 64, 4, [0, 10])
    r = P.Rope(16, torch.zeros(8))
    Q, K = torch.zeros(1, 10, 4, 64), torch.zeros(1, 10, 2, 64)
    with pytest.raises(ValueError, match="GPU tensor"):
        P.ecokv_prefill_rope(Q, K, s, r, None, torch.zeros_like(Q), torch.zeros_like(K))
    with pytest.raises(ValueError, match="Q or K"):
        P.ecokv_prefill_rope(None, None, s, r)
    pool = torch.zeros(1, 3, 2, 16, 64)
    with pytest.raises(ValueError, match="GPU tensor"):
        P.ecokv_append(Q, K, K, s, r, torch.zeros(10, dtype=torch.int32), None, torch.zeros(10, dtype=torch.int32),
                       P.Tails(pool, pool.clone(), torch.zeros(10, 2, dtype=torch.int32)), Q)
    with pytest.raises(ValueError, match="GPU tensor"):
        P.ecokv_decode_shared(torch.zeros(1, 4, 1, 64), torch.zeros(5, 64), torch.zeros(5, 64), s, [0, 1], torch.zeros(2, dtype=torch.int32),
                              torch.zeros(2, dtype=torch.int32), 5, None, None, 0, torch.zeros(256))
    with pytest.raises(ValueError, match="one entry per prompt"):
        P.ecokv_decode_shared_workspace_size(s, [0, 1, 2], 5, 0)
    with pytest.raises(ValueError):
        P.Tails(pool[0], pool[0], torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.Tails(pool, pool, torch.zeros(1, dtype=torch.int32))
