"""Sums over many positions in the 4-bit cache's attention: what many small probabilities
add up to next to a few large ones.

Tolerances, before any run.  Probabilities enter the product as halves, 2^7 or more where
the row's largest (of those a reference covers) is: 11 bits, 2^-11 of each at most, and
below 2^-21 of the largest half a step of the smallest halves, 2^-25 / 2^7 = 2^-32 of the
largest.  The scores' and the sums' roundings in fp32: 2^-18 of the result for exponents up
to 27 (27 ln 2 2^-24, the exponential's 2^-22, sums of up to 4,096 equal terms taken in
tiles).  Outputs lie between the roundings of both ends of what that allows.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_kv4 import f64, flags, i32, pkg

pytestmark = pytest.mark.gpu

SINKS = (0, 32, 64, 96)        # one for each warp that takes chunks of 32 in turn


def stored(k, v, page):
    """A cache of one sequence with these keys and values [n, n_kv, hd], and its table row."""
    n, nkv, hd = k.shape
    pages = -(-n // page)
    cache = pkg().KV4Cache.empty(pages, page, nkv, hd)
    rope = pkg().buddy_rope_table(2, hd, 1e4)
    cache.buddy_kv4_append(None, k, v, i32(np.zeros(n)), torch.arange(n, device="cuda"), rope, None)   # no rotation at 0
    return cache, torch.arange(pages, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("w", [10.3, 14.9, 20.3, 23.42, 24.7, 26.6])
@pytest.mark.parametrize("m,batch", [(1, 700), (4, 350), (40, 200)])
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_attention_adds_up_small_probabilities(w, m, batch, out_dtype):
    """Four positions with the largest score, 4,092 with 2^-w of their probability each."""
    n, nq, hd = 4096, 4, 64
    k, v = torch.zeros(2, n, 1, hd, device="cuda")
    k[list(SINKS), 0, 0] = 7.0                     # stored exactly: scale 1, code 15
    v[:, 0, 1] = 7.0
    v[list(SINKS), 0, 1] = 0.0
    cache, row = stored(k, v, 64)
    table = row.expand(batch, -1).contiguous()     # all sequences read the same pages
    q = torch.zeros(batch * m, nq, hd, device="cuda", dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    scale = float(np.float32(w * math.log(2) / 7))
    out, fl = torch.full((batch * m, nq, hd), 77.0, device="cuda", dtype=out_dtype), flags()
    cache.buddy_kv4_attention(q, i32([n] * batch), table, out, i32(np.arange(batch + 1) * m), m, scale, fl)
    assert fl.item() == 0
    count = n - m + 1 + np.tile(np.arange(m), batch) - len(SINKS)
    tail = math.exp(-7 * scale)
    total = len(SINKS) + count * tail
    want = 7 * count * tail / total
    tol = want * (2.0 ** -11 + 2.0 ** -18) + 7 * count * 2.0 ** -32 / total
    got = f64(out)
    lo, hi = (f64(torch.as_tensor(x).to(out_dtype))[:, None] for x in (want - tol, want + tol))
    assert np.all((got[:, :, 1] >= lo) & (got[:, :, 1] <= hi)), (np.abs(got[:, :, 1] / want[:, None] - 1)).max()
    assert not got[:, :, 2:].any() and not got[:, :, 0].any()


# ------------------------------------------------------------------ every position, once
# Queries of zeros weigh all positions alike, and values are whole numbers: the sums of
# 2^7 v and of 2^7 are exact (below 2^24 in steps of 2^7, the exponential of a whole number is
# exact), so that an output is its mean but for the division's two roundings: 2^-22 of it.  A
# position left out or counted twice changes all of a row's outputs by about 1 / n of them.
def rand_lens(lo, hi, count, seed):
    return [int(x) for x in np.random.default_rng(seed).integers(lo, hi, count)]


LENS = {"65536": [65536], "120001": [120001], "two": [9000, 13000], "mixed": [3000, 20, 6000, 17, 5000, 0, 1],
        "chunk-ends": [32 * k + d for k in (1, 2, 3, 12, 13, 24, 40) for d in (-1, 0, 1)],
        "700-short": rand_lens(0, 90, 700, 1), "250-of-50-200": rand_lens(50, 200, 250, 2),
        "250-of-30-1000": rand_lens(30, 1000, 250, 3), "33-of-900": rand_lens(800, 1000, 33, 4)}


def whole_numbers(lens, page, nkv, hd, seed):
    """A cache of sequences with values of -7 .. 7, its table, and the values of each."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    total, held = sum(lens), [-(-n // page) for n in lens]
    v = torch.randint(-7, 8, (total, nkv, hd), generator=g, device="cuda").float()
    v[:, :, ::32] = 7.0                            # the largest of each 32 makes the scale 1
    k = torch.randn(total, nkv, hd, generator=g, device="cuda")
    ids = torch.randperm(sum(held) + 2, generator=g, device="cuda").int()
    table = torch.full((len(lens), max(held) + 1), -1, device="cuda", dtype=torch.int32)
    slots, at = [], 0
    for i, (n, h) in enumerate(zip(lens, held)):
        table[i, :h] = ids[at:at + h]
        p = torch.arange(n, device="cuda")
        slots.append(table[i].long()[p // page] * page + p % page)
        at += h
    cache = pkg().KV4Cache.empty(sum(held) + 2, page, nkv, hd)
    cache.buddy_kv4_append(None, k, v, i32(np.zeros(total)), torch.cat(slots), pkg().buddy_rope_table(2, hd, 1e4), None)
    return cache, table, v.split(lens)


@pytest.mark.parametrize("name", list(LENS))
@pytest.mark.parametrize("heads,page", [((8, 2, 64), 16), ((2, 2, 128), 64), ((8, 1, 128), 128), ((7, 7, 64), 32),
                                        ((6, 2, 128), 16)])
@pytest.mark.parametrize("m", [1, 2, 7, 40])
def test_attention_counts_every_position_once(name, heads, page, m):
    nq, nkv, hd = heads
    lens = LENS[name]
    cache, table, vals = whole_numbers(lens, page, nkv, hd, len(lens))
    n_new = [m if m == 1 else (i * 5 + m) % (m + 1) for i in range(len(lens))]
    n_new[0] = m
    starts = np.concatenate([[0], np.cumsum(n_new)])
    q = torch.zeros(starts[-1], nq, hd, device="cuda", dtype=torch.bfloat16)
    out, fl = torch.full((starts[-1], nq, hd), 77.0, device="cuda"), flags()
    cache.buddy_kv4_attention(q, i32(lens), table, out, i32(starts), m, flags=fl)
    assert fl.item() == 0
    for i, (n, mi, v) in enumerate(zip(lens, n_new, vals)):
        if not mi:
            continue
        sums = torch.cat([torch.zeros(1, nkv, hd, device="cuda", dtype=torch.float64), v.double().cumsum(0)])
        seen = torch.arange(n - mi + 1, n + 1, device="cuda").clamp(min=0)
        want = (sums[seen] / seen.clamp(min=1)[:, None, None]).repeat_interleave(nq // nkv, 1)
        got = out[starts[i]:starts[i + 1]].double()
        assert torch.all((got - want).abs() <= want.abs() * 2.0 ** -22), (i, n, mi, ((got - want).abs() / want.abs()).max())
