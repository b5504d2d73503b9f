"""The paged 4-bit cache's attention on streams other than the current one, and in graphs,
with the workspaces that the cache makes for itself.

Results are compared bit by bit with those of the same call by itself: the order of all
sums is fixed."""
import numpy as np
import pytest
import torch

from test_gpu_kv4 import i32, make_cache, pkg

pytestmark = pytest.mark.gpu


def fresh(cache):
    """The same pages behind a new handle, which has no workspace yet."""
    return pkg().KV4Cache(cache.k_pages, cache.v_pages, cache.page_size)


def make(n, n_new, nq=8, seed=0):
    cache, table, _ = make_cache([n], 64, 2, 64, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(n_new, nq, 64, generator=g, device="cuda").bfloat16()
    rows, kv = i32([0, n_new]), i32([n])

    def call(c, out, **kw):
        c.buddy_kv4_attention(q, kv, table, out, rows, n_new, **kw)

    want = torch.empty_like(q)
    call(fresh(cache), want)
    torch.cuda.synchronize()
    return cache, call, want


def keep_busy(ms=40):
    """Work on the current stream that outlasts what the test enqueues behind and beside it."""
    x = torch.randn(4096, 4096, device="cuda")
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    y = x @ x
    b.record()
    b.synchronize()
    for _ in range(int(ms / max(a.elapsed_time(b), 1e-3)) + 1):
        y = x @ x
    return y


@pytest.mark.parametrize("n_new", [1, 3, 70])
def test_first_call_on_another_stream_does_not_wait_for_the_current_one(n_new):
    cache, call, want = make(20011, n_new)
    side = torch.cuda.Stream()
    c, out = fresh(cache), torch.full_like(want, 7)
    torch.cuda.synchronize()
    keep_busy()
    call(c, out, stream=side)
    call(c, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_a_larger_workspace_on_another_stream():
    cache, few, want_few = make(9000, 1)
    _, many, want_many = make(9000, 100)
    side = torch.cuda.Stream()
    c, o1, o2 = fresh(cache), torch.full_like(want_few, 7), torch.full_like(want_many, 7)
    torch.cuda.synchronize()
    keep_busy()
    for _ in range(3):
        few(c, o1, stream=side)
        many(c, o2, stream=side)
    side.synchronize()
    assert torch.equal(o1, want_few) and torch.equal(o2, want_many)


def test_streams_share_a_cache_without_waiting_for_each_other():
    cache, call, want = make(30000, 1)
    streams = [torch.cuda.Stream() for _ in range(3)]
    c = fresh(cache)
    outs = [[torch.full_like(want, 7) for _ in range(40)] for _ in streams]
    torch.cuda.synchronize()
    for k in range(40):
        for s, out in zip(streams, outs):
            if k % 2:
                call(c, out[k], stream=s)
            else:
                with torch.cuda.stream(s):
                    call(c, out[k])
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(o, want) for o in out)


def test_captured_calls_want_a_workspace():
    cache, call, want = make(20011, 1)
    side = torch.cuda.Stream()
    c, out = fresh(cache), torch.full_like(want, 7)
    call(c, out, stream=side)                 # the stream's own workspace is not for its graphs
    ws = torch.zeros(c.workspace_bytes(8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(ValueError, match="workspace"):
            call(c, out)
        call(c, out, workspace=ws)
    out.fill_(7)
    eager = torch.full_like(want, 7)
    torch.cuda.synchronize()
    for _ in range(20):                       # replays next to eager calls of the same cache
        graph.replay()
        call(c, eager, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(eager, want)
