"""The handles Rope and Tails on the host: a tensor replaced between calls is the
one that the next call is given, with its sizes.  (The binding's argument check,
which takes GPU tensors only, is replaced by one that takes the CPU's.)"""
import ctypes

import pytest
import torch


@pytest.fixture
def E(monkeypatch):
    from paper_2609_06663_amd import ecokv as E

    def arg(t, name, dtypes, numel, device, optional=False):
        if t is None:
            assert optional, name
            return None
        if t.dtype not in dtypes:
            raise TypeError(name)
        assert t.numel() >= numel, name
        return t.data_ptr()

    monkeypatch.setattr(E, "_arg", arg)
    return E


def pool(pages, H=2, page=16, D=64, L=1, dtype=torch.bfloat16):
    return torch.zeros(L, pages, H, page, D, dtype=dtype)


def shape(E, L=1, H=2, D=64):
    return E.Shape(L, 2 * H, H, D, 4, [0, 10])


def test_tails_follow_their_tensors(E):
    t = E.Tails(pool(6), pool(6), torch.zeros(3, 2, dtype=torch.int32))
    s = shape(E)
    assert ctypes.addressof(t._arg(s, torch.bfloat16, None)._obj) == ctypes.addressof(t.c)
    t.table = torch.zeros(5, 4, dtype=torch.int32)       # more continuations, longer ones
    t._arg(s, torch.bfloat16, None)
    assert t.c.table == t.table.data_ptr() and (t.c.num_conts, t.c.max_pages) == (5, 4)
    t.K = pool(20)                                       # a larger pool: K, then V
    t.V = pool(20)
    t._arg(s, torch.bfloat16, None)
    assert (t.c.K, t.c.V, t.c.num_pages, t.c.page_size) == (t.K.data_ptr(), t.V.data_ptr(), 20, 16)
    t.K, t.V = pool(40, page=8), pool(40, page=8)
    t._arg(s, torch.bfloat16, None)
    assert (t.c.num_pages, t.c.page_size) == (40, 8)


def test_tails_refuse_replacements_that_do_not_fit(E):
    t = E.Tails(pool(6), pool(6), torch.zeros(3, 2, dtype=torch.int32))
    s = shape(E)
    t._arg(s, torch.bfloat16, None)
    t.K = pool(7)                                        # V is still the old one
    with pytest.raises(ValueError, match="two tensors"):
        t._arg(s, torch.bfloat16, None)
    t.V = pool(7)
    t.table = torch.zeros(6, dtype=torch.int32)
    with pytest.raises(ValueError, match="num_conts"):
        t._arg(s, torch.bfloat16, None)
    t.table = torch.zeros(3, 2, dtype=torch.int32)
    t._arg(s, torch.bfloat16, None)
    t.K, t.V = pool(7, dtype=torch.float32), pool(7, dtype=torch.float32)
    with pytest.raises(TypeError):
        t._arg(s, torch.bfloat16, None)
    t.K, t.V = pool(7, H=3), pool(7, H=3)
    with pytest.raises(ValueError, match="3 KV heads"):
        t._arg(s, torch.bfloat16, None)


def test_rope_follows_its_tensors(E):
    w = lambda v: torch.full((64,), v, dtype=torch.bfloat16)
    r = E.Rope(32, torch.zeros(16))
    r._arg(64, torch.bfloat16, None)
    assert r.c.q_norm is None and r.c.k_norm is None
    r.freq = torch.ones(16)
    r.q_norm, r.k_norm = w(2.0), w(3.0)
    r._arg(64, torch.bfloat16, None)
    assert (r.c.freq, r.c.q_norm, r.c.k_norm) == (r.freq.data_ptr(), r.q_norm.data_ptr(), r.k_norm.data_ptr())
    r.q_norm = None
    r._arg(64, torch.bfloat16, None)
    assert r.c.q_norm is None and r.c.k_norm == r.k_norm.data_ptr()
    r.freq = torch.ones(4, dtype=torch.float64)
    with pytest.raises(TypeError):
        r._arg(64, torch.bfloat16, None)


def test_numbers_past_32_bits_are_refused():
    # (ctypes cuts them to 32 bits: a bound of 2^32 would be one of 0, and the rows left out)
    import paper_2609_06663_amd as P
    s = P.Shape(1, 4, 2, 64, 4, [0, 10, 30])
    size = lambda fan=(0, 1, 3), mc=5, mt=7: P.ecokv_decode_shared_workspace_size(s, list(fan), mc, mt)
    assert size() > 0
    for big in (2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 64 + 5, -2 ** 31 - 1, -2 ** 32 + 5):
        for kw in (dict(fan=(0, 1, big)), dict(fan=(0, big, 3)), dict(fan=(big, 1, 3)), dict(mc=big), dict(mt=big)):
            with pytest.raises(ValueError, match="32 bits"):
                size(**kw)
        with pytest.raises(ValueError, match="32 bits"):
            P.Rope(big, torch.zeros(8))
        with pytest.raises(ValueError, match="32 bits"):
            P.ecokv_rope_freqs(16, 10000.0, big)
    with pytest.raises(ValueError, match="32 bits"):
        P.ecokv_rope_freqs(-2 ** 32 + 16)
    size(mc=2 ** 31 - 1, mt=2 ** 31 - 1)
