"""What a draft, a commit and their accumulated weights read on another stream than
the one that its memory came from: the allocator is told, and what a captured graph
reads is kept.  The library's calls are replaced by recorders, the tensors are the
CPU's and say that they are not."""
import gc
import weakref

import pytest
import torch

from test_drafts_host import i32, made, rec, tokens  # noqa: F401  (rec: a fixture)


class Device(torch.Tensor):
    """A tensor of the CPU that records the streams it was recorded on."""

    is_cuda = True

    def record_stream(self, s):
        self.__dict__.setdefault("streams", []).append(s)


def device(t):
    return t.as_subclass(Device)


@pytest.fixture
def current(rec, monkeypatch):  # noqa: F811
    state = {"capturing": False}
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: rec.current)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["capturing"])
    return state


def drafted(co, stream):
    t = co.tree([-1, 0])
    for name in ("masks", "steps", "conts"):
        setattr(t, name, device(getattr(t, name)))
    co.draft(*tokens(6), t, stream=stream)
    return t


@pytest.mark.parametrize("stream", ["s", None])
def test_what_is_read_is_recorded(current, stream):
    co, want = made(), [stream or "current"]
    t = drafted(co, stream)
    for x in (t.masks, t.steps, t.conts):
        assert x.streams == want
    path, acc = device(i32([[0, 1]] * 3)), device(i32([1] * 3))
    co.commit(path, acc)
    co.accumulate()
    assert path.streams == 2 * want and acc.streams[0] == want[0] and set(acc.streams) == set(want)


@pytest.mark.parametrize("capturing", [False, True])
def test_a_captured_tree_is_kept(current, capturing):
    co = made()
    current["capturing"] = capturing
    t = weakref.ref(drafted(co, "s"))
    gc.collect()
    assert (t() is not None) == capturing
