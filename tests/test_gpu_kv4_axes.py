"""Rotation by several position axes (buddy_qk_norm_rope and buddy_kv4_append with axes).

A frequency is turned by one position with the arithmetic of the calls with one axis, so every
channel equals, bit by bit, that of a call whose only positions are those of its axis.
Against the float64 oracle the tolerances are those of the calls with one axis: 2^-20 of a
pair's length, and 2^-8 of a value (half a step) where it is rounded to bf16."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from test_gpu_kv4 import BAD_PAGE, BAD_POSITION, EPS, HEADS, THETA, f64, flags, make_rows, pkg, read

pytestmark = pytest.mark.gpu

LAYOUTS = {64: [((8, 12, 12), False), ((12, 10, 10), True), ((16, 16), False), ((5, 9, 9, 9), True), ((32,), False),
                ((0, 1, 31), False), ((7, 0, 20, 5), False)],
           128: [((16, 24, 24), False), ((24, 20, 20), True), ((32, 32), True), ((10, 20, 14, 20), False), ((64,), True),
                 ((1, 0, 0, 63), True)]}


def places(n_axes, T, max_pos, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, max_pos, (n_axes, T), generator=g, device="cuda", dtype=torch.int32)


def turn(q, k, pos, rope, gain, axes=None, fl=None):
    qo, ko = torch.full_like(q.contiguous(), 7), torch.full_like(k.contiguous(), 7)
    pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, *gain, EPS, fl, axes=axes)
    return qo, ko


def composed(q, k, pos, rope, gain, axes):
    """The same from calls with one axis."""
    h = q.shape[-1] // 2
    axis = torch.tensor(list(axes.axis)[:h], device="cuda").repeat(2)
    out = [torch.full_like(x.contiguous(), 7) for x in (q, k)]
    for a in range(axes.n_axes):
        for o, one in zip(out, turn(q, k, pos[a].contiguous(), rope, gain)):
            o[..., axis == a] = one[..., axis == a]
    return out


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 130])
def test_every_frequency_turns_by_its_axis(heads, dtype, T):
    for n, (sections, turns) in enumerate(LAYOUTS[heads[2]]):
        q, k, _, _, rope, gain = make_rows(T, heads, dtype, seed=T + n, gains=n % 2 == 0)
        axes = pkg().buddy_rope_axes(heads[2], sections, turns)
        pos, fl = places(len(sections), T, 600, n), flags()
        got = turn(q, k, pos, rope, gain, axes, fl)
        for x, y in zip(got, composed(q, k, pos, rope, gain, axes)):
            assert torch.equal(x, y), (sections, turns)
        assert fl.item() == 0
        for x, src, g in zip(got, (q, k), gain):
            want = O.norm_rope_axes(f64(src), None if g is None else f64(g), f64(pos), list(axes.axis), THETA, EPS)
            h = want.shape[-1] // 2
            pair = np.tile(np.sqrt(want[..., :h] ** 2 + want[..., h:] ** 2), 2)
            tol = pair * 2.0 ** -20 + 1e-30 + (np.abs(want) * 2.0 ** -8 if dtype == torch.bfloat16 else 0)
            assert np.all(np.abs(f64(x) - want) <= tol)


@pytest.mark.parametrize("heads,T", [((32, 8, 128), 4001), ((9, 3, 64), 4097), ((32, 8, 128), 820)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tokens_in_place(heads, T, dtype):
    q, k, _, _, rope, gain = make_rows(T, heads, dtype, seed=T)
    sections, turns = LAYOUTS[heads[2]][T % 2]
    axes, pos = pkg().buddy_rope_axes(heads[2], sections, turns), places(3, T, 600)
    want = composed(q, k, pos, rope, gain, axes)
    pkg().buddy_qk_norm_rope(q, k, pos, rope, q, k, *gain, EPS, axes=axes)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_text_is_turned_as_with_one_axis():
    q, k, _, pos, rope, gain = make_rows(40, (6, 2, 128), torch.bfloat16)
    want = turn(q, k, pos, rope, gain)
    for sections, turns in LAYOUTS[128]:
        axes = pkg().buddy_rope_axes(128, sections, turns)
        # one row for all axes, without a copy of it
        got = turn(q, k, pos[None].expand(len(sections), -1), rope, gain, axes)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_positions_in_rows_of_a_larger_table():
    q, k, _, _, rope, gain = make_rows(21, (4, 2, 64), torch.float32)
    axes, table = pkg().buddy_rope_axes(64, (8, 12, 12)), places(5, 300, 600)
    want = turn(q, k, table[1:4, 40:61].contiguous(), rope, gain, axes)
    got = turn(q, k, table[1:4, 40:61], rope, gain, axes)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("heads", [(9, 3, 64), (32, 8, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 77, 3001])
def test_append(heads, dtype, T):
    nq, nkv, hd = heads
    for sections, turns in LAYOUTS[hd][:2]:
        q, k, v, _, rope, gain = make_rows(T, heads, dtype, seed=T)
        axes, pos = pkg().buddy_rope_axes(hd, sections, turns), places(3, T, 600, T)
        page, n_pages = 32, T // 32 + 3
        slot = torch.randperm(n_pages * page, device="cuda")[:T].contiguous()
        cache, plain = (pkg().KV4Cache.empty(n_pages, page, nkv, hd) for _ in range(2))
        qo, ko = torch.full_like(q.contiguous(), 7), torch.full_like(k.contiguous(), 7)
        fl = flags()
        cache.buddy_kv4_append(q, k, v, pos, slot, rope, qo, *gain, EPS, fl, k_out=ko, axes=axes)
        want = turn(q, k, pos, rope, gain, axes)
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1]) and fl.item() == 0
        # values are stored as without axes; keys, in fp32, as values that equal them are
        zero = torch.zeros(T, dtype=torch.int32, device="cuda")
        plain.buddy_kv4_append(None, k, v, zero, slot, rope, None)
        assert torch.equal(cache.v_pages, plain.v_pages)
        if dtype == torch.float32:
            plain.buddy_kv4_append(None, ko, ko, zero, slot, rope, None)
            assert torch.equal(read(cache, slot)[0], read(plain, slot)[1])


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_tokens_that_are_left_out(axis):
    """A position that is negative, or past the tables, on any axis."""
    heads = (4, 2, 64)
    q, k, v, _, rope, gain = make_rows(6, heads, torch.bfloat16)
    axes, pos = pkg().buddy_rope_axes(64, (8, 12, 12)), places(3, 6, 600)
    good = turn(q, k, pos, rope, gain, axes)
    for value, flag in ((-1, 0), (600, BAD_POSITION), (2 ** 31 - 1, BAD_POSITION), (-2 ** 31, 0)):
        bad = pos.clone()
        bad[axis, 2] = value
        fl = flags()
        got = turn(q, k, bad, rope, gain, axes, fl)
        assert fl.item() == flag
        for g, w in zip(got, good):
            assert torch.all(g[2] == 7)
            keep = [0, 1, 3, 4, 5]
            assert torch.equal(g[keep], w[keep])
        cache = pkg().KV4Cache.empty(2, 16, 2, 64)
        cache.k_pages.fill_(0x5A)
        before = cache.k_pages.clone()
        fl.zero_()
        cache.buddy_kv4_append(None, k[2:3], v[2:3], bad[:, 2:3], torch.zeros(1, dtype=torch.int64, device="cuda"), rope,
                               None, flags=fl, axes=axes)
        assert fl.item() == flag and torch.equal(cache.k_pages, before)


def test_slots_that_are_not_there():
    q, k, v, _, rope, gain = make_rows(3, (4, 2, 64), torch.float32)
    axes, pos = pkg().buddy_rope_axes(64, (8, 12, 12)), places(3, 3, 600)
    cache, fl = pkg().KV4Cache.empty(2, 16, 2, 64), flags()
    slot = torch.tensor([5, 32, -1], device="cuda")
    qo = torch.full_like(q.contiguous(), 7)
    cache.buddy_kv4_append(q, k, v, pos, slot, rope, qo, *gain, EPS, fl, axes=axes)
    assert fl.item() == BAD_PAGE and torch.equal(qo, turn(q, k, pos, rope, gain, axes)[0])
    assert cache.v_pages.count_nonzero() <= 2 * 36


def test_no_tokens():
    q, k, v, _, rope, gain = make_rows(2, (4, 2, 64), torch.float32)
    axes = pkg().buddy_rope_axes(64, (8, 12, 12))
    none = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    turn(q[:0], k[:0], none, rope, gain, axes)
    pkg().KV4Cache.empty(2, 16, 2, 64).buddy_kv4_append(q[:0], k[:0], v[:0], none, torch.empty(0, dtype=torch.int64, device="cuda"),
                                                       rope, q[:0], axes=axes)


def test_a_graph_and_another_stream():
    q, k, _, _, rope, gain = make_rows(9, (6, 2, 128), torch.bfloat16)
    axes, pos = pkg().buddy_rope_axes(128, (24, 20, 20), True), places(3, 9, 600)
    qo, ko = torch.full_like(q.contiguous(), 7), torch.full_like(k.contiguous(), 7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, *gain, EPS, stream=side, axes=axes)
    torch.cuda.current_stream().wait_stream(side)
    want = turn(q, k, pos, rope, gain, axes)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, *gain, EPS, axes=axes)
    pos.copy_(places(3, 9, 600, 5))
    graph.replay()
    want = turn(q, k, pos, rope, gain, axes)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
