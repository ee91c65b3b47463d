"""pipeline.Continuations on the host: which stream its calls go to and which
calls it refuses.  The library's calls are replaced by recorders, the tensors
are the CPU's."""
import contextlib

import pytest
import torch


class Recorder:
    """Stands for the library and for torch's current stream."""

    def __init__(self, monkeypatch):
        from paper_2609_06663_amd import pipeline
        self.current, self.calls = "current", []
        monkeypatch.setattr(pipeline.torch.cuda, "stream", self.stream)
        monkeypatch.setattr(pipeline.E, "ecokv_append", lambda *a: self.calls.append(("append", a[-1] or self.current)))
        monkeypatch.setattr(pipeline.E, "ecokv_decode_shared", lambda *a: self.calls.append(("decode_shared", a[-1] or self.current)))

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s or self.current
        yield
        self.current = before

    def counters(self, co):
        """Its counters, whose increments are recorded with the stream they go to."""
        rec, at = self, co._at

        class Counters:
            def add_(self, v):
                rec.calls.append(("advance", rec.current))
                at.add_(v)

        co._at = Counters()


def continuations(fan_out=(3, 2)):
    import paper_2609_06663_amd as P
    from paper_2609_06663_amd.pipeline import Continuations, EvictionPass
    ep = EvictionPass(P.Shape(1, 4, 2, 64, 4, [0, 40, 100]), [20, 30], device="cpu", dtype=torch.float32)
    return Continuations(ep, list(fan_out), 3, P.Rope(0), 4)


def tokens(n, layers=1):
    return [torch.zeros(layers, n, h, 64) for h in (4, 2, 2)]


def test_advance_is_on_the_stream_of_the_step(monkeypatch):
    rec = Recorder(monkeypatch)
    co = continuations()
    rec.counters(co)
    co.step(*tokens(5), stream="s")
    co.advance()
    co.step(*tokens(5))
    co.advance()
    assert rec.calls == [("append", "s"), ("decode_shared", "s"), ("advance", "s"),
                         ("append", "current"), ("decode_shared", "current"), ("advance", "current")]
    assert co.length == 2 and co.rows.tolist() == [2] * 5 and co.tail_counts.tolist() == [3] * 5
    assert co.positions.tolist() == [42] * 3 + [62] * 2


def test_advance_takes_a_stream(monkeypatch):
    rec = Recorder(monkeypatch)
    co = continuations()
    rec.counters(co)
    co.step(*tokens(5), stream="s")
    co.advance(stream="t")
    assert rec.calls[-1] == ("advance", "t")


def test_a_step_takes_one_token_of_every_continuation(monkeypatch):
    # fewer would leave Q_dec, which the attention reads, laid out for fewer
    rec = Recorder(monkeypatch)
    co = continuations()
    for n in (0, 1, 4, 6):
        with pytest.raises(ValueError, match="5 continuations"):
            co.step(*tokens(n))
    with pytest.raises(ValueError, match="5 continuations"):
        co.step(*(t[0, 0] for t in tokens(5)))
    assert rec.calls == []
    co.step(*(t[0] for t in tokens(5)))  # (one layer: without its dimension)
    assert len(rec.calls) == 2
