"""What the 4-bit cache's Python class does around its calls, without a GPU: the
library and the streams are stand-ins."""
import contextlib

import pytest
import torch

from paper_2606_09514_gb300 import binding as b


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Library:
    """Notes the workspace of every attention call; `capturing`: handles of streams under capture."""

    def __init__(self, current):
        self.current, self.capturing, self.calls = current, set(), []

    def buddy_kv4_attention_workspace(self, n_q, n_kv, hd, max_new):
        return 64 * n_q * max_new

    def call_stream_for_workspace(self, q, stream):
        handle = (stream or self.current).cuda_stream
        if handle in self.capturing:
            raise ValueError("workspace: a call that is captured in a graph wants one given")
        return handle

    def call_kv4_attention(self, *args):
        stream, workspace = args[-1], args[-2]
        self.calls.append(((stream or self.current).cuda_stream, workspace))
        return b.BUDDY_OK


@pytest.fixture
def cache(monkeypatch):
    """A cache of a stand-in library whose zeroed memory knows the stream that zeroes it."""
    lib = Library(Stream(0))
    now = [lib.current]

    @contextlib.contextmanager
    def on(stream):
        now.append(stream or now[-1])
        yield
        now.pop()

    made = []
    real = torch.zeros

    def zeros(*size, **kw):
        t = real(*size, **kw)
        made.append((now[-1].cuda_stream, t))
        return t

    monkeypatch.setattr(b.torch.cuda, "stream", on)
    monkeypatch.setattr(b.torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(b.torch, "zeros", zeros)
    monkeypatch.setattr(b, "load_library", lambda *a: lib)
    monkeypatch.setattr(b, "_vectors", lambda *a: None)
    c = b.KV4Cache(*(torch.empty(4, 2, 16 * 36, dtype=torch.uint8) for _ in range(2)), 16)
    return c, lib, made


def attend(c, n_new=1, **kw):
    q = torch.empty(3, 4, 64)
    c.buddy_kv4_attention(q, None, None, q, None, n_new, **kw)


def test_a_workspace_is_zeroed_on_the_stream_of_its_calls(cache):
    c, lib, made = cache
    side = Stream(7)
    for n_new, stream in ((1, None), (1, side), (5, side), (5, None), (2, side), (2, None)):
        attend(c, n_new, stream=stream)
    zeroed_on = {id(t): s for s, t in made}
    assert len(lib.calls) == 6
    for handle, ws in lib.calls:
        assert zeroed_on[id(ws)] == handle
        assert ws.dtype == torch.uint8
    # a larger one where it is needed, and no new one where not
    assert len(made) == 4
    assert lib.calls[2][1] is lib.calls[4][1] and lib.calls[3][1] is lib.calls[5][1]


def test_streams_have_workspaces_of_their_own(cache):
    c, lib, _ = cache
    streams = [None, Stream(7), Stream(8)]
    for _ in range(2):
        for s in streams:
            attend(c, stream=s)
    assert len({id(ws) for _, ws in lib.calls}) == 3


def test_a_captured_call_wants_a_workspace(cache):
    c, lib, made = cache
    side = Stream(9)
    attend(c, stream=side)                 # also where there is one already: a replay shares it with nobody
    lib.capturing.add(9)
    n = len(made)
    with pytest.raises(ValueError, match="workspace"):
        attend(c, stream=side)
    assert len(made) == n and len(lib.calls) == 1
    ws = torch.zeros(1024, dtype=torch.uint8)
    attend(c, stream=side, workspace=ws)
    assert lib.calls[-1][1] is ws
    attend(c)                              # another stream's is not taken from the graph's
    assert lib.calls[-1][1] is not ws


def test_a_given_workspace_is_used(cache):
    c, lib, made = cache
    c.workspace = torch.zeros(1024, dtype=torch.uint8)
    n = len(made)
    attend(c)
    attend(c, stream=Stream(3))
    assert len(made) == n and all(ws is c.workspace for _, ws in lib.calls)


# ------------------------------------------------------------------ rotary tables
def test_rotary_tables_are_filled_on_the_stream_that_they_are_made_on(monkeypatch):
    """Memory of another stream's pool may still be in use there."""
    now, made, filled = [Stream(0)], {}, []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream or now[-1])
        yield
        now.pop()

    real = torch.empty

    def empty(*size, device, **kw):
        t = real(*size, **kw)
        made[t.data_ptr()] = (now[-1].cuda_stream, device)
        return t

    class Lib:
        def buddy_rope_table(self, co, si, max_pos, hd, theta, stream):
            filled.append((made[co.value], made[si.value], stream.value or 0))
            return b.BUDDY_OK

    monkeypatch.setattr(b.torch.cuda, "stream", on)
    monkeypatch.setattr(b.torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(b.torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(b.torch, "empty", empty)
    monkeypatch.setattr(b, "load_library", lambda *a: Lib())
    for stream, want in ((None, 0), (Stream(7), 7)):
        co, si = b.buddy_rope_table(9, 64, 1e4, stream=stream)
        assert co.shape == si.shape == (9, 32)
        (co_on, _), (si_on, _), launched = filled[-1]
        assert co_on == si_on == launched == want


@pytest.mark.parametrize("device", ["cpu", "meta", torch.device("cpu")])
def test_rotary_tables_are_on_a_gpu(monkeypatch, device):
    class Lib:
        def buddy_rope_table(self, *args):
            raise AssertionError("called with host memory")

    monkeypatch.setattr(b, "load_library", lambda *a: Lib())
    with pytest.raises(ValueError, match="device"):
        b.buddy_rope_table(9, 64, 1e4, device)
