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
