"""Calls of so many tokens that a team of lanes takes several heads: crossing from queries to
keys to values, with a short last group, in place.  Their results equal, bit by bit, those of
calls of a hundred tokens, where a team has one head."""
import pytest
import torch

from test_gpu_kv4 import EPS, check_turned, flags, make_rows, pkg

pytestmark = pytest.mark.gpu

# heads of a team: tokens x heads / 16,384 (kv4_rows.cu), up to eight
NORMS = [((32, 8, 128), 820), ((32, 8, 128), 1300), ((32, 8, 128), 4001), ((9, 3, 64), 2731), ((9, 3, 64), 4097),
         ((9, 3, 64), 11003), ((5, 1, 64), 9000)]
APPENDS = [((32, 8, 128), 700), ((32, 8, 128), 1100), ((32, 8, 128), 3001), ((9, 3, 64), 2185), ((9, 3, 64), 3277),
           ((9, 3, 64), 8801), ((4, 4, 64), 7000)]


def pieces(T, step=100):
    return [slice(t, min(T, t + step)) for t in range(0, T, step)]


@pytest.mark.parametrize("heads,T", NORMS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gains", [True, False])
def test_norm_of_many_tokens(heads, T, dtype, gains):
    q, k, _, pos, rope, gain = make_rows(T, heads, dtype, seed=T, gains=gains)
    q0, k0, q1, k1 = (torch.full_like(x.contiguous(), 7) for x in (q, k, q, k))
    fl = flags()
    for s in pieces(T):
        pkg().buddy_qk_norm_rope(q[s], k[s], pos[s], rope, q0[s], k0[s], *gain, EPS, fl)
    some = pos[:50]
    check_turned(q0[:50], q[:50], gain[0], some, dtype)
    check_turned(k0[:50], k[:50], gain[1], some, dtype)
    pkg().buddy_qk_norm_rope(q, k, pos, rope, q1, k1, *gain, EPS, fl)
    assert torch.equal(q0, q1) and torch.equal(k0, k1)
    pkg().buddy_qk_norm_rope(q, k, pos, rope, q, k, *gain, EPS, fl)        # in place, in rows shared with the values
    assert torch.equal(q0, q) and torch.equal(k0, k) and fl.item() == 0


@pytest.mark.parametrize("heads,T", APPENDS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_of_many_tokens(heads, T, dtype):
    nq, nkv, hd = heads
    q, k, v, pos, rope, gain = make_rows(T, heads, dtype, seed=T)
    pos[3], pos[T - 2] = -1, -5
    page, n_pages = 64, T // 64 + 3
    slot = torch.randperm(n_pages * page, device="cuda")[:T].contiguous()
    slot[7], slot[T - 1] = -1, -3
    a, b, c = (pkg().KV4Cache.empty(n_pages, page, nkv, hd) for _ in range(3))
    q0, k0, q1, k1 = (torch.full_like(x.contiguous(), 7) for x in (q, k, q, k))
    fl = flags()
    for s in pieces(T):
        a.buddy_kv4_append(q[s], k[s], v[s], pos[s], slot[s], rope, q0[s], *gain, EPS, fl, k_out=k0[s])
    b.buddy_kv4_append(q, k, v, pos, slot, rope, q1, *gain, EPS, fl, k_out=k1)
    assert torch.equal(q0, q1) and torch.equal(k0, k1)
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages) and a.v_pages.any()
    assert torch.all(q1[3] == 7) and torch.all(k1[T - 2] == 7)
    left = v.clone()
    c.buddy_kv4_append(q, k, v, pos, slot, rope, q, *gain, EPS, fl, k_out=k)     # in place
    q0[3], q0[T - 2], k0[3], k0[T - 2] = q[3], q[T - 2], k[3], k[T - 2]           # (tokens that are left out)
    assert torch.equal(q0, q) and torch.equal(k0, k) and torch.equal(v, left) and fl.item() == 0
    assert torch.equal(a.k_pages, c.k_pages) and torch.equal(a.v_pages, c.v_pages)


def test_special_keys():
    """At position 0 the rotation multiplies by one and zero: keys are stored as values are, but
    for NaN and infinities, which make NaN of the channel that they are turned with."""
    hd, page = 64, 16
    x = torch.zeros(7, 1, hd, device="cuda")
    x[1, 0, 3] = float("nan")
    x[2, 0, 5], x[2, 0, 6] = float("inf"), 3.0
    x[3] = 2.0 ** -30
    x[4, 0, 0], x[4, 0, 1] = 7 * 2.0 ** -24, -3 * 2.0 ** -24
    x[5, 0, 0] = 1e30
    x[6, 0, 0], x[6, 0, 33], x[6, 0, 40] = 7.0, -2.5, 1.25
    cache = pkg().KV4Cache.empty(2, page, 1, hd)
    slot = torch.arange(3, 10, device="cuda")
    cache.buddy_kv4_append(None, x, x, torch.zeros(7, dtype=torch.int32, device="cuda"), slot,
                           pkg().buddy_rope_table(8, hd, 1e4), None)
    k, v = (torch.empty(7, 1, hd, device="cuda") for _ in range(2))
    cache.buddy_kv4_read(slot, k, v)
    k, v = k[:, 0].cpu(), v[:, 0].cpu()
    same = [0, 3, 4, 5, 6]
    assert torch.equal(k[same], v[same]) and torch.isfinite(v[same]).all() and v[6].any() and v[5, 0] == 6272
    assert torch.isnan(k[1]).all()
    assert torch.isnan(v[1, :32]).all() and torch.all(v[1, 32:] == 0)
    assert k[2, 5] == v[2, 5] == 6272 and k[2, :32].count_nonzero() == 1 and v[2].count_nonzero() == 1
    assert torch.isnan(k[2, 32:]).all()
