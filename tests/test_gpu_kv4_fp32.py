"""The 4-bit cache's attention with fp32 queries or fp32 outputs.

Tolerance, before any run, as the 2-norm of a sequence's error over that of its outputs.
Query elements and probabilities enter with 22 bits (2^-22 each); a score is summed in fp32
over 2 hd / 16 products of 16, 2^-24 of it each (2^-20 for hd 128), and is 16 at most
here after its scale: 2^-16 of a probability where all of that went one way, 2^-18 as it
does not; an output is summed over 2 n / 16 products, 2^-24 each, which do not go one way
either: 2^-19 for 3,000 positions.  Together below 2^-16.  (Eleven bits give some 2^-12.)
"""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from test_gpu_kv4 import f64, flags, i32, make_cache

pytestmark = pytest.mark.gpu
F, B = torch.float32, torch.bfloat16
LENS = [1, 33, 500, 3000, 0, 127, 128, 1000, 20]


def check(heads, page, lens, n_new, dtype, out_dtype, up=1.0, amp=1.0, seed=0):
    nq, nkv, hd = heads
    cache, table, vals = make_cache(lens, page, nkv, hd, seed=seed)
    starts = np.concatenate([[0], np.cumsum(n_new)])
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (amp * up * torch.randn(starts[-1], nq, hd, generator=g, device="cuda")).to(dtype)
    out, fl = torch.full((starts[-1], nq, hd), 77.0, device="cuda", dtype=out_dtype), flags()
    scale = hd ** -0.5 / up
    cache.buddy_kv4_attention(q, i32(lens), table, out, i32(starts), max(n_new), scale, fl)
    assert fl.item() == 0
    for i, (n, m) in enumerate(zip(lens, n_new)):
        if not m:
            continue
        want = O.attention(f64(q[starts[i]:starts[i] + m]), *vals[i], m, scale)
        got = f64(out[starts[i]:starts[i] + m])
        if out_dtype is B:                          # the rounding is known: both ends of the tolerance, rounded
            off = 2.0 ** -16 * np.linalg.norm(want)
            lo, hi = (f64(torch.as_tensor(x).to(B)) for x in (want - off, want + off))
            assert np.all((got >= lo) & (got <= hi)), (i, n, m)
        else:
            err = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
            assert err <= 2.0 ** -16, (i, n, m, err)


@pytest.mark.parametrize("heads,page", [((8, 2, 64), 16), ((6, 2, 128), 64), ((8, 1, 128), 128), ((7, 7, 64), 32),
                                        ((32, 8, 128), 64)])
@pytest.mark.parametrize("m", [1, 2, 5, 60])
@pytest.mark.parametrize("dtype,out_dtype", [(F, F), (B, F), (F, B)])
def test_attention_in_fp32(heads, page, m, dtype, out_dtype):
    n_new = [m if m == 1 else (3 * i + m) % (m + 1) for i in range(len(LENS))]
    n_new[3] = m
    check(heads, page, LENS, n_new, dtype, out_dtype, seed=m)


@pytest.mark.parametrize("up", [2.0 ** 40, 2.0 ** -40, 2.0 ** -110])
@pytest.mark.parametrize("m", [1, 4, 60])
def test_attention_in_fp32_of_large_and_small_queries(up, m):
    """The scale takes the power of two back: the same scores."""
    check((8, 2, 64), 16, [300, 64, 1000], [m, m, 1], F, F, up)


@pytest.mark.parametrize("m", [1, 200])
def test_attention_in_fp32_behind_a_long_prefix(m):
    check((8, 2, 128), 64, [20011, 300], [m, m], F, F)
    check((4, 4, 64), 64, [16384], [m], F, F)


@pytest.mark.parametrize("up", [2.0 ** 40, 2.0 ** -12, 2.0 ** -20, 2.0 ** -40, 2.0 ** -110])
@pytest.mark.parametrize("m", [1, 4, 60])
def test_attention_in_bf16_of_large_and_small_queries(up, m):
    """A power of two in all queries, taken back by the scale, changes no bit; in every other head's, it
    leaves both kinds of rows within what bf16 calls are held to (2^-11 + 2^-12 of the largest value, and the
    output's rounding of 2^-8).  Rows of zeros and of one element are among them."""
    lens, n_new = [300, 64, 1000], [m, m, 1]
    cache, table, vals = make_cache(lens, 16, 2, 64)
    starts = np.concatenate([[0], np.cumsum(n_new)])
    g = torch.Generator(device="cuda").manual_seed(m)
    # two bits per element: whole as halves whatever the row's power of two is
    q = torch.randint(-3, 4, (starts[-1], 8, 64), generator=g, device="cuda").to(B) / 2
    q[0, 0], q[-1, 3] = 0.0, 0.0
    q[-1, 3, 9] = 1.5

    def call(x, scale):
        out = torch.full_like(q, 77.0)
        cache.buddy_kv4_attention(x, i32(lens), table, out, i32(starts), m, scale)
        return out

    assert torch.equal(call((q.float() * up).to(B), 0.125 / up), call(q, 0.125))
    some = torch.arange(8, device="cuda")[:, None] % 2 == 0
    x = (q.float() * torch.where(some, up, 1.0)).to(B)
    for heads, scale in ((slice(0, None, 2), 0.125 / up), (slice(1, None, 2), 0.125)):
        got = f64(call(x, scale))
        for i, (n, mi) in enumerate(zip(lens, n_new)):
            rows = slice(starts[i], starts[i + 1])
            want = O.attention(f64(q[rows]), *vals[i], mi, 0.125)
            tol = np.abs(vals[i][1]).max() * (2.0 ** -11 + 2.0 ** -12) + np.abs(want) * 2.0 ** -8
            assert np.all((np.abs(got[rows] - want) <= tol)[:, heads]), (i, heads)
