"""Attention over selected pages of the 4-bit cache: bounds, selection, attention.

Bounds are values that the cache holds: they equal the oracle's.  Selections follow from sums
in a stated order: they equal those of the same sums in numpy's fp32.  Attention has the
tolerances of buddy_kv4_attention (test_gpu_kv4.py)."""
import functools

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from test_gpu_kv4 import BAD_PAGE, BAD_POSITION, at_once, f64, flags, i32, make_cache, pkg

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def starts_of(n_new):
    return np.concatenate([[0], np.cumsum(n_new)])


def same(a, b):
    """Equal, NaN where NaN."""
    np.testing.assert_array_equal(f64(a) if isinstance(a, torch.Tensor) else a, b)


# ------------------------------------------------------------------ bounds
LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 511, 1000]


def check_bounds(cache, table, lens, n_new, keys=None, rows=True):
    """The touched pages' bounds; the others' stay."""
    P, hd = cache.page_size, cache.head_dim
    bounds = cache.empty_bounds().fill_(7)
    want = f64(bounds)
    held = O.entries(cache.k_pages.cpu().numpy(), P, hd) if keys is None else keys
    ids = table.cpu().numpy()
    for i, (n, m) in enumerate(zip(lens, n_new)):
        for j in range(max(0, n - m) // P, -(-n // P) if m else 0):
            if 0 <= ids[i, j] < len(want):
                want[ids[i, j]] = O.page_bounds(held[ids[i, j]][None], P, min(P, n - j * P))[0]
    fl = flags()
    for _ in range(2):
        cache.buddy_kv4_bounds(bounds, i32(lens), table, i32(starts_of(n_new)) if rows else None,
                               max(n_new) if rows else 1, fl)
        same(bounds, want)
    return fl.item()


@pytest.mark.parametrize("heads", [(2, 64), (1, 64), (3, 64), (8, 128), (1, 128), (7, 128)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_bounds(heads, page):
    nkv, hd = heads
    cache, table, _ = make_cache(LENGTHS, page, nkv, hd, seed=page)
    assert check_bounds(cache, table, LENGTHS, [1] * len(LENGTHS), rows=False) == 0
    assert check_bounds(cache, table, LENGTHS, [(7 * i) % 5 for i in range(len(LENGTHS))]) == 0
    assert check_bounds(cache, table, LENGTHS, [n // (1 + i % 3) for i, n in enumerate(LENGTHS)]) == 0
    assert check_bounds(cache, table, LENGTHS, [n + i % 4 for i, n in enumerate(LENGTHS)]) == 0     # more than there are


def test_bounds_of_special_keys():
    """NaN scales inside the sequence, negative scales, zeros, the largest values."""
    nkv, hd, page = 1, 64, 16
    cache, table, _ = make_cache([40], page, nkv, hd)
    held = O.entries(cache.k_pages.cpu().numpy(), page, hd)
    codes = torch.as_tensor(O.unpack(cache.k_pages[:, :, :page * hd // 2].cpu().numpy().reshape(-1, nkv, page, hd // 2)))
    scales = torch.ones(len(held), nkv, page, 2)
    ids = table[0].tolist()
    scales[ids[0], 0, 3, 1] = float("nan")
    scales[ids[0], 0, 5, 0] = 896.0
    scales[ids[1]] = 0.0
    scales[ids[2], 0, 2, 0] = -0.25
    scales[ids[2], 0, 8:] = float("nan")         # behind the end
    cache.k_pages.copy_(torch.as_tensor(O.blocks(codes.numpy(), scales.numpy())))
    assert check_bounds(cache, table, [40], [40]) == 0
    bounds = cache.empty_bounds()
    cache.buddy_kv4_bounds(bounds, i32([40]), table, i32([0, 40]), 40)
    assert torch.isnan(bounds[ids[0], 0, :, 32:]).all() and not torch.isnan(bounds[ids[0], 0, :, :32]).any()
    assert not bounds[ids[1]].any() and not torch.isnan(bounds[ids[2]]).any()


def test_bounds_leave_bad_sequences_and_pages_out():
    nkv, hd, page = 2, 64, 16
    lens = [40, 33, 20, 50]
    cache, table, _ = make_cache(lens, page, nkv, hd)
    held = O.entries(cache.k_pages.cpu().numpy(), page, hd)
    n_pages = len(held)
    for bad in (-1, n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[1, 2], t[2, 1] = bad, bad
        assert check_bounds(cache, t, lens, [4, 20, 1, 7], held) == BAD_PAGE
    bounds = cache.empty_bounds().fill_(7)
    for kv, rows, max_new, alive in (([40, -1, 20, 50], [0, 1, 2, 3, 4], 1, [0, 2, 3]),
                                     ([40, 33, 20, table.shape[1] * page + 1], [0, 1, 2, 3, 4], 1, [0, 1, 2]),
                                     ([40, 33, 20, 50], [0, 1, 5, 4, 5], 2, [0, 3]),
                                     ([40, 33, 20, 50], [-1, 1, 2, 3, 4], 2, [1, 2, 3]),
                                     ([40, 33, 20, 50], [0, 1, 2, 5, 6], 2, [0, 1, 3])):
        fl = flags()
        bounds.fill_(7)
        cache.buddy_kv4_bounds(bounds, i32(kv), table, i32(rows), max_new, fl)
        assert fl.item() == BAD_POSITION
        touched = {int(table[i, (lens[i] - 1) // page]) for i in alive}
        assert {int(p) for p in torch.nonzero((bounds != 7).flatten(1).any(1)).flatten()} == touched


def test_bounds_at_offsets_past_32_bits():
    nkv, hd, page = 8, 128, 128
    first = 2 ** 32 // (nkv * page * 72) + 5
    cache, table, vals = make_cache([300], page, nkv, hd, first_page=first)
    assert cache.k_pages.numel() > 2 ** 32
    bounds = torch.full((cache.k_pages.shape[0], nkv, 2, hd), 7, dtype=torch.float16, device="cuda")
    cache.buddy_kv4_bounds(bounds, i32([300]), table, i32([0, 300]), 300)
    k = vals[0][0]
    for j in range(3):
        got, mine = f64(bounds[int(table[0, j])]), k[:, j * page:(j + 1) * page]
        np.testing.assert_array_equal(got[:, 0], mine.min(1))
        np.testing.assert_array_equal(got[:, 1], mine.max(1))


# ------------------------------------------------------------------ selection
def make_select(lens, n_new, page, heads, dtype, seed=0, pad=0, max_pages=None, levels=None):
    """Random bounds and a table; no page is looked at, so the cache has one byte pattern.
    levels: so many different values of the bounds, for equal scores."""
    nq, nkv, hd = heads
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    row = max_pages or max(need + [1]) + 1
    n_pages = sum(need) + 3
    ids = rng.permutation(n_pages)
    table = np.full((len(lens), row), -1)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = ids[at:at + n]
        at += n
    cache = pkg().KV4Cache.empty(n_pages, page, nkv, hd)
    g = torch.Generator(device="cuda").manual_seed(seed)
    mid = torch.randn(n_pages, nkv, 1, hd, generator=g, device="cuda")
    if levels:
        mid = torch.randint(0, levels, (n_pages, nkv, 1, 1), generator=g, device="cuda").float().expand(-1, -1, 1, hd)
    bounds = torch.cat([mid - 1, mid + 1], 2).half()
    T = sum(n_new) + pad
    q = torch.randn(T, nq, hd, generator=g, device="cuda").to(dtype)
    return cache, i32(table), bounds, q


def want_pages(q, bounds, table, lens, n_new, page, budget, first, last, T):
    """Lists and lengths in numpy."""
    q, bounds, table = (x.float().cpu().numpy() if x.is_floating_point() else x.cpu().numpy() for x in (q, bounds, table))
    nkv = bounds.shape[1]
    pages, visible = np.full((T, nkv, budget), -1), np.full(T, -1)
    at = 0
    for i, (n, m) in enumerate(zip(lens, n_new)):
        for j in range(m):
            t, p = at + j, n - m + j
            if p < 0:
                visible[t] = 0
                continue
            N = p // page + 1
            ids = table[i, :N]
            there = (ids >= 0) & (ids < len(bounds))
            score = O.page_scores(q[t], bounds[np.where(there, ids, 0)])
            for g in range(nkv):
                s = [x if ok else None for x, ok in zip(score[g], there)]
                sel = O.select(s, budget, first, last)
                pages[t, g, :len(sel)] = ids[sel]
            visible[t] = (min(N, budget) - 1) * page + p % page + 1
        at += m
    return pages, visible


def check_select(cache, table, bounds, q, lens, n_new, budget, first=1, last=1, rows=True, flag=0):
    T, n = q.shape[0], sum(n_new)
    pages = torch.full((T, cache.n_kv, budget), 55, dtype=torch.int32, device="cuda")
    visible = torch.full((T,), 55, dtype=torch.int32, device="cuda")
    fl = flags()
    cache.buddy_kv4_select(q, bounds, i32(lens), table, pages, visible, i32(starts_of(n_new)) if rows else None,
                           max(n_new) if rows else 1, first, last, fl)
    wp, wv = want_pages(q, bounds, table, lens, n_new, cache.page_size, budget, first, last, T)
    np.testing.assert_array_equal(visible.cpu().numpy(), wv)
    np.testing.assert_array_equal(pages[:n].cpu().numpy(), wp[:n])
    assert torch.all(pages[n:] == 55)          # rows behind the last sequence
    assert fl.item() == flag
    return pages, visible


@pytest.mark.parametrize("heads", [(4, 2, 64), (5, 1, 64), (9, 3, 64), (16, 2, 128), (7, 7, 128), (6, 2, 128)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 128])
def test_select_single_tokens(heads, dtype, page):
    lens = [page * n + d for n, d in ((0, 0), (0, 1), (1, -1), (1, 0), (1, 1), (4, 0), (5, 0), (5, 1), (9, 3), (40, -2), (131, 7))]
    made = make_select(lens, [1] * len(lens), page, heads, dtype, seed=page)
    for budget in (1, 2, 5, 33):
        check_select(*made, lens, [1] * len(lens), budget, 0 if budget == 1 else 1, 1, rows=budget % 2 == 1)


@pytest.mark.parametrize("budget,first,last", [(1, 0, 1), (7, 0, 1), (7, 3, 4), (7, 3, 3), (7, 0, 7), (8, 6, 1), (64, 2, 30),
                                               (200, 1, 1), (3, 1, 1)])
def test_select_first_and_last_pages(budget, first, last):
    lens = [16 * 20 + 3, 5, 16 * 7, 16 * 8 + 1, 16 * 70, 16 * 300 - 1]
    made = make_select(lens, [1] * 6, 16, (4, 2, 64), torch.bfloat16, seed=budget)
    check_select(*made, lens, [1] * 6, budget, first, last)


@pytest.mark.parametrize("dtype", DTYPES)
def test_select_several_tokens(dtype):
    """Proposed tokens, prompts, more tokens than positions, empty sequences, rows behind the last."""
    lens, n_new = [100, 0, 333, 7, 64, 2, 500, 31], [3, 0, 40, 7, 1, 5, 130, 0]
    made = make_select(lens, n_new, 16, (6, 2, 64), dtype, seed=3, pad=9)
    for budget in (2, 6, 40):
        check_select(*made, lens, n_new, budget)


@pytest.mark.parametrize("lens,n_new", [([16 * 3000 - 3, 16 * 700, 16 * 8000], [3, 1, 6]), ([16 * 9001 - 1, 16 * 30], [2, 3]),
                                        ([16 * 500, 16 * 130 + 2, 16 * 90, 16 * 260], [4, 9, 2, 5])])
def test_select_several_tokens_of_many_pages(lens, n_new):
    """Tokens that share a walk over thousands of pages, and tables too long for that."""
    for heads, dtype in (((2, 1, 64), torch.bfloat16), ((3, 1, 128), torch.float32)):
        made = make_select(lens, n_new, 16, heads, dtype, seed=len(lens))
        for budget in (3, 80, 500):
            check_select(*made, lens, n_new, budget)


def test_select_several_tokens_special_scores():
    """Ties, NaN, and pages that are not there, for tokens that share a walk."""
    lens, n_new = [16 * 90, 16 * 300 + 5, 16 * 40], [3, 6, 2]
    cache, table, bounds, q = make_select(lens, n_new, 16, (4, 2, 64), torch.bfloat16, seed=2, levels=3)
    for budget in (5, 31, 85):
        check_select(cache, table, bounds, q, lens, n_new, budget)
    bounds[table[1, 7].long(), 0, 0, 3] = float("nan")
    q[1] = float("nan")
    table[0, 5], table[1, 100], table[2, 3] = -1, 10 ** 7, -9
    for budget in (5, 30):
        check_select(cache, table, bounds, q, lens, n_new, budget, flag=BAD_PAGE)


def test_select_by_clusters_in_a_graph():
    lens = [16 * 1000 - 2]
    cache, table, bounds, q = make_select(lens, [1], 16, (4, 2, 128), torch.bfloat16)
    pages, visible = torch.empty(1, 2, 30, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    kv_len = i32(lens)
    graph = torch.cuda.CUDAGraph()
    cache.buddy_kv4_select(q, bounds, kv_len, table, pages, visible)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for _ in range(3):
            cache.buddy_kv4_select(q, bounds, kv_len, table, pages, visible)
    for n in (16 * 1000 - 2, 16 * 31, 16 * 500 + 1, 5):
        q.copy_(torch.randn_like(q))
        kv_len.fill_(n)
        pages.fill_(55)
        graph.replay()
        wp, wv = want_pages(q, bounds, table, [n], [1], 16, 30, 1, 1, 1)
        np.testing.assert_array_equal(pages.cpu().numpy(), wp)
        assert visible.item() == wv[0]


@pytest.mark.parametrize("levels", [1, 2, 5])
def test_select_ties_go_to_the_lower_position(levels):
    lens = [16 * 50, 16 * 300 + 1, 16 * 1000]
    made = make_select(lens, [1] * 3, 16, (2, 2, 64), torch.bfloat16, seed=levels, levels=levels)
    for budget in (4, 17, 256, 299):
        check_select(*made, lens, [1] * 3, budget)


def test_select_many_pages():
    """Up to the largest table there may be."""
    for n_pages in (255, 256, 257, 4095, 10001, 40000):
        lens = [n_pages * 16 - 5, 16 * 40]
        made = make_select(lens, [1, 1], 16, (2, 1, 64), torch.bfloat16, seed=n_pages, max_pages=n_pages)
        for budget in (3, 64, 3000 if n_pages > 3000 else 100, n_pages - 1):
            check_select(*made, lens, [1, 1], budget)


@pytest.mark.parametrize("heads", [(4, 2, 128), (2, 1, 64), (24, 8, 128)])
@pytest.mark.parametrize("n_pages", [127, 128, 129, 255, 256, 257, 700, 1100, 2100])
def test_select_by_clusters(heads, n_pages):
    """One token, or few: the pages of a head shared by 1 to 16 CTAs, of which the last may have none."""
    for lens in ([n_pages * 16 - 1], [n_pages * 16 - 15, 16 * 90 + 4, 3], [n_pages * 16] * 20):
        made = make_select(lens, [1] * len(lens), 16, heads, torch.bfloat16, seed=n_pages, max_pages=n_pages)
        check_select(*made, lens, [1] * len(lens), 40, rows=len(lens) == 3)


def test_select_of_scores_near_and_far():
    """Scores in one binade, in many, and alike but for a few bits."""
    lens = [16 * 1500]
    cache, table, bounds, q = make_select(lens, [1], 16, (2, 2, 64), torch.float32, seed=1)
    for scale in (1e-30, 1e-3, 1e4):
        q[0] = 0
        q[0, :, 5] = scale
        wide = torch.randn(bounds.shape[:2], device="cuda")
        for spread in (1.0, 1e-3, 30.0):
            bounds[:, :, 1, 5] = (1000 + spread * wide if spread != 30.0 else 10 ** (4 * torch.rand_like(wide))).half()
            for budget in (3, 65, 1400):
                check_select(cache, table, bounds, q, lens, [1], budget)


@pytest.mark.parametrize("batch", [31, 33, 1025, 3000])
def test_select_finds_each_tokens_sequence(batch):
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 200, batch)]
    n_new = [int(x) for x in rng.integers(0, 3, batch) * (rng.random(batch) < 0.6)]
    n_new[0] = 2
    made = make_select(lens, n_new, 16, (2, 1, 64), torch.bfloat16, seed=batch, pad=4)
    check_select(*made, lens, n_new, 4)


def test_select_special_scores():
    """NaN bounds and queries come first, infinities in their order, pages that are not there last."""
    lens = [16 * 60] * 3
    cache, table, bounds, q = make_select(lens, [1] * 3, 16, (4, 2, 64), torch.float32, seed=9)
    ids = table.cpu().numpy()
    bounds[ids[0, 7], 0, 0, 3] = float("nan")
    bounds[ids[0, 50], 0, 1, 60] = float("nan")
    bounds[ids[0, 20], 1, 1] = float("inf")
    bounds[ids[0, 21], 1, 0] = float("-inf")
    bounds[ids[0, 30], 1] = float("-inf")
    q[1, 2] = 3e38                       # sums that overflow
    q[2, 0, 0] = float("nan")            # every page of head 0: the first ones
    for budget in (3, 4, 5, 40):
        check_select(cache, table, bounds, q, lens, [1] * 3, budget)
    q[2, 0, 0] = float("-inf")
    q[2, 1, 1] = float("inf")
    check_select(cache, table, bounds, q, lens, [1] * 3, 9)
    table[0, 5], table[0, 6], table[1, 59], table[1, 0], table[2, 4] = -1, 10 ** 6, -7, 2 ** 31 - 1, bounds.shape[0]
    for budget in (3, 20, 58, 59):
        check_select(cache, table, bounds, q, lens, [1] * 3, budget, flag=BAD_PAGE)
    check_select(cache, table, bounds, q, lens, [1] * 3, 60)          # all pages: none is looked at


def test_select_in_bad_sequences():
    lens = [16 * 9] * 4
    cache, table, bounds, q = make_select(lens, [1] * 4, 16, (4, 2, 64), torch.bfloat16, max_pages=10)
    for kv, rows, max_new, n_tok, alive in (([144, -1, 144, 144], [0, 1, 2, 3, 4], 1, 4, {0, 2, 3}),
                                            ([144, 161, 144, 144], [0, 1, 2, 3, 4], 1, 4, {0, 2, 3}),
                                            ([144] * 4, [0, 1, 3, 4, 4], 1, 4, {0, 3}),
                                            ([144] * 4, [0, 1, 2, 3, 5], 2, 4, {0, 1, 2}),
                                            ([144] * 4, [2, 2, 2, 3, 4], 2, 4, {2, 3}),
                                            ([144] * 4, [0, 4, 1, 3, 4], 4, 4, None)):
        pages = torch.full((n_tok, 2, 3), 55, dtype=torch.int32, device="cuda")
        visible = torch.full((n_tok,), 55, dtype=torch.int32, device="cuda")
        fl = flags()
        cache.buddy_kv4_select(q, bounds, i32(kv), table, pages, visible, i32(rows), max_new, flags=fl)
        v = visible.cpu().tolist()
        if alive is None:            # row starts that do not ascend: whatever, within the buffers
            assert set(v) <= {-1, 48, 47, 46, 45, 33, 40}
            continue
        assert {t for t in range(n_tok) if v[t] == 48} == alive and all(v[t] == -1 for t in range(n_tok) if t not in alive)
        assert fl.item() == (0 if rows[0] == 2 else BAD_POSITION)
        for t in range(n_tok):
            assert (pages[t] == 55).all() == (t not in alive)


def test_select_bounds_scores():
    """A score is a bound: the heads' largest products with a page's keys add up to no more (but for
    the fp32 sums: 128 terms of at most 4 x 3 x 0.5 x 7 each, off by less than 2^-24 x 128 x 42 a sum)."""
    lens, page = [3008], 32
    cache, table, _ = make_cache(lens, page, 2, 64)
    bounds = cache.empty_bounds()
    cache.buddy_kv4_bounds(bounds, i32(lens), table, i32([0, 3008]), 3008)
    keys = O.entries(cache.k_pages.cpu().numpy(), page, 64)
    q = torch.randn(1, 8, 64, device="cuda")
    score = O.page_scores(q[0].cpu().numpy(), bounds[table[0, :94].long()].cpu().numpy())
    for g in range(2):
        top = np.einsum("hd,npd->hnp", f64(q[0, 4 * g:4 * g + 4]), keys[table[0, :94].cpu().numpy()][:, g])
        assert np.all(top.max(-1).sum(0) <= score[g] + 1e-3)


# ------------------------------------------------------------------ attention
def lists_for(lens, table, page, nkv, budget, seed=0):
    """Random lists: ascending pages of each sequence, its last always; their positions."""
    rng = np.random.default_rng(seed)
    ids = table.cpu().numpy()
    pages, visible, at = np.full((len(lens), nkv, budget), -1), np.zeros(len(lens), int), []
    for t, n in enumerate(lens):
        N = -(-n // page)
        k = min(N, budget)
        mine = []
        for g in range(nkv):
            j = np.sort(rng.permutation(max(0, N - 1))[:max(0, k - 1)]).tolist() + ([N - 1] if N else [])
            pages[t, g, :k] = ids[t, j]
            mine.append(j)
        visible[t] = (k - 1) * page + (n - 1) % page + 1 if n else 0
        at.append(mine)
    return i32(pages), i32(visible), at


def check_pages(cache, lens, vals, pages, visible, at, nq, dtype=torch.bfloat16, out_dtype=torch.bfloat16, scale=0.0, amp=1.5,
                strided=False, seed=0, drop=(), flag=0):
    """drop: (token, head, entry) of lists whose page is not there."""
    hd, nkv, P, T = cache.head_dim, cache.n_kv, cache.page_size, len(lens)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (amp * torch.randn(T, nq, hd, generator=g, device="cuda")).to(dtype)
    out = torch.full((T, nq, hd), 77.0, dtype=out_dtype, device="cuda")
    if strided:
        q = torch.cat([q, q], 1)[:, :nq]
        out = torch.cat([out, out], 1)[:, nq:]
    fl = flags()
    for _ in range(2):
        before = out.clone()
        out.fill_(77.0)
        cache.buddy_kv4_attention_pages(q, visible, pages, out, scale, fl)
    assert torch.equal(out, before) and fl.item() == flag
    got, sc, G = f64(out), scale or 1 / np.sqrt(hd), nq // nkv
    vis = visible.cpu().numpy()
    for t in range(T):
        if vis[t] < 0:
            assert np.all(got[t] == 77)
            continue
        for h in range(nkv):
            pos = np.array([j * P + x for e, j in enumerate(at[t][h]) for x in range(P)
                            if e * P + x < vis[t] and (t, h, e) not in drop], int)
            k, v = (x[h][pos][None] for x in vals[t])
            qi = f64(q[t:t + 1, h * G:(h + 1) * G])
            want = O.attention(qi, k, v, 1, sc)
            top = np.abs(v).max(initial=0.0)
            tol = top * (2.0 ** -11 + 2.0 ** -12) + np.abs(want) * (2.0 ** -8 if out_dtype == torch.bfloat16 else 2.0 ** -22)
            if dtype == torch.float32 and len(pos):
                tol = tol + top * 2 * np.expm1(2.0 ** -11 * sc * (np.abs(qi[0]) @ np.abs(k[0]).T).max())
            err = np.abs(got[t, h * G:(h + 1) * G] - want[0])
            assert np.all(err <= tol), (t, h, (err / np.maximum(tol, 1e-30)).max())
    return q, out


@pytest.mark.parametrize("heads", [(4, 2, 64), (5, 1, 64), (8, 1, 128), (7, 7, 128), (14, 2, 128), (9, 3, 64)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention(heads, page):
    nq, nkv, hd = heads
    cache, table, vals = make_cache(LENGTHS, page, nkv, hd, seed=page)
    for budget in (1, 3, 9):
        check_pages(cache, LENGTHS, vals, *lists_for(LENGTHS, table, page, nkv, budget, seed=budget), nq)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
def test_attention_types_scales_strides(dtype, out_dtype, hd, page):
    lens = [5, 130, 0, 777]
    cache, table, vals = make_cache(lens, page, 2, hd)
    lists = lists_for(lens, table, page, 2, 4)
    for scale, strided in ((0.0, False), (0.3, True)):
        check_pages(cache, lens, vals, *lists, 6, dtype, out_dtype, scale, strided=strided)
    check_pages(cache, lens, vals, *lists, 6, dtype, out_dtype, amp=40.0)


@pytest.mark.parametrize("lens,budget", [([30011], 400), ([30011, 9000, 20], 200), ([4000] * 40, 30), ([700] * 500, 3),
                                         ([2000] * 33, 31)])
def test_attention_shares(lens, budget):
    """Lists that many CTAs share, and many short ones."""
    if len(lens) == 500:
        lens = [int(x) for x in np.random.default_rng(0).integers(0, 700, 500)]
    cache, table, vals = make_cache(lens, 16 if budget > 3 else 64, 2, 64, seed=len(lens))
    check_pages(cache, lens, vals, *lists_for(lens, table, cache.page_size, 2, budget), 8)


def many(n, seed=0):
    """n lengths: LENGTHS over and over in any order."""
    return [LENGTHS[i % len(LENGTHS)] for i in np.random.default_rng(seed).permutation(n)]


@pytest.mark.parametrize("heads,n", [((4, 2, 64), 300), ((5, 1, 64), 600), ((8, 1, 128), 520), ((7, 7, 128), 80),
                                     ((14, 2, 128), 260), ((9, 3, 64), 180), ((3, 1, 128), 1000)])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_attention_of_many_lists(heads, n, page):
    """So many lists that warps take them alone; some are cut between warps."""
    nq, nkv, hd = heads
    lens = many(n, page)
    cache, table, vals = make_cache(lens, page, nkv, hd, seed=page)
    for budget in (1, 5, 40):
        check_pages(cache, lens, vals, *lists_for(lens, table, page, nkv, budget, seed=budget), nq)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_of_many_lists_types(dtype, out_dtype, hd):
    lens = many(260)
    cache, table, vals = make_cache(lens, 16, 2, hd)
    lists = lists_for(lens, table, 16, 2, 20)
    check_pages(cache, lens, vals, *lists, 10, dtype, out_dtype, 0.3, strided=True)
    check_pages(cache, lens, vals, *lists, 10, dtype, out_dtype, amp=40.0)


@pytest.mark.parametrize("long", [30011, 6000])
def test_attention_of_long_lists_among_many(long):
    """A list that a hundred warps share, next to short ones and to tokens that are left out."""
    lens = many(270)
    lens[3], lens[70], lens[269] = long, long - 16, 17
    cache, table, vals = make_cache(lens, 16, 2, 64)
    pages, visible, at = lists_for(lens, table, 16, 2, long // 16 + 1)
    visible[5], visible[80], visible[71] = -1, -1, 0
    check_pages(cache, lens, vals, pages, visible, at, 16)


def test_many_lists_without_some_pages():
    lens = many(260)
    cache, table, vals = make_cache(lens, 16, 2, 64)
    pages, visible, at = lists_for(lens, table, 16, 2, 12)
    rng = np.random.default_rng(4)
    drop = [(t, h, e) for t in range(260) for h in range(2) for e in range(12) if e * 16 < visible[t] and rng.random() < 0.3]
    for x, d in enumerate(drop):
        pages[d] = (-1, cache.k_pages.shape[0], 2 ** 31 - 1, -2 ** 31)[x % 4]
    check_pages(cache, lens, vals, pages, visible, at, 4, drop=set(drop), flag=BAD_PAGE)
    q, out, fl = torch.randn(260, 4, 64, device="cuda"), torch.full((260, 4, 64), 77.0, device="cuda"), flags()
    visible[150] = 12 * 16 + 1
    cache.buddy_kv4_attention_pages(q, visible, pages, out, flags=fl)
    assert fl.item() == BAD_PAGE | BAD_POSITION and torch.all(out[150] == 77) and not torch.any(out[149] == 77)


def test_no_list_at_all():
    """Every token left out: nothing is written, and the workspace stays as it is."""
    cache, table, vals = make_cache([50] * 600, 16, 1, 64)
    pages, visible, at = lists_for([50] * 600, table, 16, 1, 2)
    cache.workspace = torch.zeros(cache.workspace_bytes(4), dtype=torch.uint8, device="cuda")
    out = torch.full((600, 4, 64), 77.0, device="cuda")
    cache.buddy_kv4_attention_pages(torch.randn(600, 4, 64, device="cuda"), torch.full_like(visible, -1), pages, out)
    assert torch.all(out == 77) and not cache.workspace.any()
    check_pages(cache, [50] * 600, vals, pages, visible, at, 4)


def test_many_lists_in_a_graph_and_on_two_streams():
    """Replays as the lists change, and two calls at once with workspaces of their own: bit by bit what
    the same call gives by itself."""
    lens = [700] * 280
    cache, table, vals = make_cache(lens, 16, 2, 64)
    q, out = torch.randn(280, 8, 64, device="cuda").bfloat16(), torch.empty(280, 8, 64, dtype=torch.bfloat16, device="cuda")
    lists = [lists_for([n] * 280, table, 16, 2, 30, seed=n)[:2] for n in (700, 33, 470, 1)]
    want = []
    for pages, visible in lists:
        want.append(torch.empty_like(out))
        cache.buddy_kv4_attention_pages(q, visible, pages, want[-1])
    torch.cuda.synchronize()
    ws = torch.zeros(cache.workspace_bytes(8), dtype=torch.uint8, device="cuda")
    pages, visible = (t.clone() for t in lists[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.buddy_kv4_attention_pages(q, visible, pages, out, workspace=ws)
    for (p, v), w in zip(lists, want):
        pages.copy_(p)
        visible.copy_(v)
        out.zero_()
        graph.replay()
        assert torch.equal(out, w)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [[torch.zeros_like(out) for _ in lists] for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for k, ((p, v), _) in enumerate(zip(lists, want)):
            for s, o in zip(streams, outs):
                cache.buddy_kv4_attention_pages(q, v, p, o[k], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for row in outs for o, w in zip(row, want))


def test_many_lists_with_nan_keys_and_values():
    """A NaN that a list's tokens see makes its outputs NaN, one behind the end does not."""
    lens = [60] * 600
    cache, table, vals = make_cache(lens, 16, 1, 64, nan_tail=False)
    pages, visible, at = lists_for(lens, table, 16, 1, 3)
    scales = [x[:, :, 16 * 32:].view(torch.float16) for x in (cache.k_pages, cache.v_pages)]
    scales[0][int(pages[3, 0, 0]), 0, 5] = float("nan")      # a key that token 3 sees
    scales[1][int(pages[8, 0, 1]), 0, 7] = float("nan")      # a value that token 8 sees
    for k in range(2):
        scales[k][int(pages[20, 0, 2]), 0, 2 * 12:] = float("nan")      # positions 60 .. 63: behind the end
    q, out = torch.randn(600, 4, 64, device="cuda"), torch.empty(600, 4, 64, device="cuda")
    cache.buddy_kv4_attention_pages(q, visible, pages, out)
    bad = torch.isnan(out).flatten(1).any(1).nonzero().flatten().tolist()
    assert bad == [3, 8] and torch.isnan(out[3]).all() and torch.isnan(out[8]).any(1).all()


def test_workspace_counters_are_left_ready():
    """Both forms over one workspace in turn: what one leaves in it the other finds."""
    lens = [900] * 300
    cache, table, vals = make_cache(lens, 16, 2, 64)
    cache.workspace = torch.zeros(cache.workspace_bytes(4), dtype=torch.uint8, device="cuda")
    for n in (300, 3, 260, 60, 256, 255):
        pages, visible, at = lists_for(lens[:n], table, 16, 2, 40)
        check_pages(cache, lens[:n], vals, pages, visible, at, 4)
        assert not cache.workspace[:8192].any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_over_all_pages_is_attention(dtype):
    """Lists of all pages: bit by bit what buddy_kv4_attention gives over the same tables."""
    lens = [5, 1300, 0, 777, 64, 2011]
    cache, table, vals = make_cache(lens, 32, 2, 128)
    pages = table[:, None].expand(-1, 2, -1).contiguous()
    q, out = check_pages(cache, lens, vals, pages, i32(lens), [[list(range(-(-n // 32)))] * 2 for n in lens], 8, dtype, dtype)
    want = torch.empty_like(out)
    cache.buddy_kv4_attention(q, i32(lens), table, want)
    assert torch.equal(out, want)


def test_attention_of_tokens_that_are_left_out():
    lens = [100, 200, 300, 50]
    cache, table, vals = make_cache(lens, 16, 2, 64)
    pages, visible, at = lists_for(lens, table, 16, 2, 5)
    visible[1], visible[3] = -1, -2 ** 31
    check_pages(cache, lens, vals, pages, visible, at, 4)
    visible[2] = 0
    check_pages(cache, lens, vals, pages, visible, at, 4)
    q, out, fl = torch.randn(4, 4, 64, device="cuda"), torch.full((4, 4, 64), 77.0, device="cuda"), flags()
    for n in (81, 2 ** 31 - 1):
        visible[0] = n                   # more than the lists hold
        cache.buddy_kv4_attention_pages(q, visible, pages, out, flags=fl)
        assert fl.item() == BAD_POSITION and torch.all(out[[0, 1, 3]] == 77) and torch.all(out[2] == 0)


@pytest.mark.parametrize("page", [16, 64])
def test_attention_without_some_pages(page):
    lens = [page * 7 + 3, page * 9, 3]
    cache, table, vals = make_cache(lens, page, 2, 64)
    pages, visible, at = lists_for(lens, table, page, 2, 5)
    drop = [(0, 0, 1), (0, 1, 4), (1, 1, 0), (1, 1, 1), (1, 1, 2), (1, 1, 3), (1, 1, 4), (2, 0, 0)]
    for d, bad in zip(drop, [-1, cache.k_pages.shape[0], 2 ** 31 - 1, -2 ** 31, -1, -5, 10 ** 6, -1]):
        pages[d] = bad
    check_pages(cache, lens, vals, pages, visible, at, 4, drop=drop, flag=BAD_PAGE)


def test_attention_of_the_same_page_twice():
    """A list is what it says: a page that it names twice counts twice."""
    lens = [64]
    cache, table, vals = make_cache(lens, 16, 1, 64)
    at = [[[2, 0, 2, 1]]]
    pages = table[:, [2, 0, 2, 1]][:, None].contiguous()
    check_pages(cache, lens, vals, pages, i32([60]), at, 4)


def test_offsets_past_32_bits():
    nkv, hd, page = 8, 128, 128
    first = 2 ** 32 // (nkv * page * 72) + 5
    lens = [700, 128]
    cache, table, vals = make_cache(lens, page, nkv, hd, first_page=first)
    assert cache.k_pages.numel() > 2 ** 32
    check_pages(cache, lens, vals, *lists_for(lens, table, page, nkv, 3), 8)


# ------------------------------------------------------------------ together
class Step:
    """A serving step as a program makes it: plan, append, bounds, selection, attention; the
    lengths advance on the GPU."""

    def __init__(self, batch, nq, nkv, hd, page, max_pages, budget, axes=None, max_new=64, dtype=torch.bfloat16):
        z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.page, self.nq, self.nkv, self.hd, self.budget, self.axes, self.dtype = page, nq, nkv, hd, budget, axes, dtype
        self.length, self.kv_len, self.rows, self.head, self.head_out = z(batch), z(batch), z(batch + 1), z(1), z(1)
        self.flags, self.table = z(1), torch.full((batch, max_pages), -1, dtype=torch.int32, device="cuda")
        n = batch * max_pages
        self.free = torch.randperm(n, device="cuda").int()
        self.cache = pkg().KV4Cache.empty(n, page, nkv, hd)
        self.cache.workspace = torch.zeros(self.cache.workspace_bytes(nq), dtype=torch.uint8, device="cuda")
        self.bounds = self.cache.empty_bounds()
        self.rope = pkg().buddy_rope_table(4096, hd, 1e4)
        self.gain = [torch.rand(hd, device="cuda") + 0.5 for _ in range(2)]

    def buffers(self, T):
        e = dict(device="cuda")
        return dict(slot=torch.empty(T, dtype=torch.int64, **e), pos=torch.empty(T, dtype=torch.int32, **e),
                    q=torch.empty(T, self.nq, self.hd, dtype=self.dtype, **e),
                    pages=torch.empty(T, self.nkv, self.budget, dtype=torch.int32, **e),
                    visible=torch.empty(T, dtype=torch.int32, **e),
                    out=torch.full((T, self.nq, self.hd), 77.0, dtype=self.dtype, **e))

    def __call__(self, x, n_new, max_new, b, grid=None, stream=None):
        nq, nkv, kw = self.nq, self.nkv, dict(flags=self.flags, stream=stream)
        pkg().buddy_page_plan(self.length, n_new, self.page, self.table, self.free, self.head, self.kv_len, self.rows,
                              b["slot"], b["pos"], self.head_out, **kw)
        self.cache.buddy_kv4_append(x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], b["pos"] if grid is None else grid,
                                    b["slot"], self.rope, b["q"], *self.gain, axes=None if grid is None else self.axes, **kw)
        self.cache.buddy_kv4_bounds(self.bounds, self.kv_len, self.table, self.rows, max_new, **kw)
        self.cache.buddy_kv4_select(b["q"], self.bounds, self.kv_len, self.table, b["pages"], b["visible"], self.rows, max_new,
                                    **kw)
        self.cache.buddy_kv4_attention_pages(b["q"], b["visible"], b["pages"], b["out"], **kw)

    def advance(self):
        self.length.copy_(self.kv_len)
        self.head.copy_(self.head_out)

    def check(self, b, n_new):
        """The call's outputs against the oracle over the entries read back."""
        assert self.flags.item() == 0
        lens, ids, P = self.kv_len.tolist(), self.table.cpu().numpy(), self.page
        held = [O.entries(x.cpu().numpy(), P, self.hd) for x in (self.cache.k_pages, self.cache.v_pages)]
        got, q, at, G = f64(b["out"]), f64(b["q"]), 0, self.nq // self.nkv
        for i, (n, m) in enumerate(zip(lens, n_new)):
            for j in range(m):
                t, p = at + j, n - m + j
                N = p // P + 1
                mine = ids[i, :N]
                score = O.page_scores(q[t], np.stack([O.page_bounds(held[0][x][None], P, min(P, n - e * P))[0]
                                                      for e, x in enumerate(mine)]))
                for g in range(self.nkv):
                    sel = O.select(list(score[g]), self.budget, 1, 1)
                    k, v = (np.concatenate([x[mine[e], g][:p + 1 - e * P] for e in sel])[None] for x in held)
                    assert b["visible"][t].item() == k.shape[1]
                    np.testing.assert_array_equal(b["pages"][t, g, :len(sel)].cpu().numpy(), mine[sel])
                    want = O.attention(q[t:t + 1, g * G:(g + 1) * G], k, v, 1, self.hd ** -0.5)
                    top = np.abs(v).max()
                    tol = top * (2.0 ** -11 + 2.0 ** -12) + np.abs(want) * 2.0 ** -8
                    assert np.all(np.abs(got[t, g * G:(g + 1) * G] - want[0]) <= tol)
            at += m


def test_a_run_as_it_is_served():
    """Prompts whose patches have three axes, in pieces next to single tokens; then single tokens by a graph."""
    torch.manual_seed(1)
    nq, nkv, hd = 6, 2, 64
    s = Step(3, nq, nkv, hd, 16, 24, 4, pkg().buddy_rope_axes(hd, (8, 12, 12)))
    for n_new in ([70, 1, 33], [40, 0, 1], [1, 16, 50], [65, 3, 1]):
        T = sum(n_new)
        x = torch.randn(T, nq + 2 * nkv, hd, device="cuda").bfloat16()
        grid = torch.randint(0, 4000, (3, T), device="cuda", dtype=torch.int32)
        b = s.buffers(T)
        s(x, i32(n_new), max(n_new), b, grid)
        s.check(b, n_new)
        s.advance()
    one, b = i32([1, 1, 1]), s.buffers(3)
    x = torch.randn(3, nq + 2 * nkv, hd, device="cuda").bfloat16()
    grid = torch.randint(0, 4000, (3, 3), device="cuda", dtype=torch.int32)
    s(x, one, 1, b, grid)
    s.check(b, [1] * 3)
    s.advance()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s(x, one, 1, b, grid)
        s.advance()
    for _ in range(20):
        x.copy_(torch.randn_like(x))
        grid.random_(0, 4000)
        graph.replay()
        s.check(b, [1] * 3)


def test_a_run_is_in_order():
    """Launches that overlap give what the same calls give with the host waiting between them."""
    outs = []
    for wait in (False, True):
        torch.manual_seed(2)
        s = Step(4, 8, 2, 128, 32, 40, 5)
        s.free = torch.arange(160, device="cuda").int()
        xs = [torch.randn(4 * m, 12, 128, device="cuda").bfloat16() for m in [200] + [1] * 30]
        bs, n = [s.buffers(len(x)) for x in xs], [i32([m] * 4) for m in [200] + [1] * 30]
        torch.cuda.synchronize()
        for x, b, m in zip(xs, bs, n):
            s(x, m, len(x) // 4, b)
            s.advance()
            if wait:
                torch.cuda.synchronize()
        outs.append([b["out"] for b in bs])
        assert s.flags.item() == 0
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_streams_of_their_own():
    """Two runs at once, each on its stream with its buffers."""
    runs = []
    for k in range(2):
        torch.manual_seed(3 + k)
        s = Step(2, 4, 2, 64, 16, 30, 3)
        s.cache.workspace = None             # the cache makes one for the stream
        xs = [torch.randn(2 * m, 8, 64, device="cuda").bfloat16() for m in [90] + [1] * 40]
        runs.append((s, xs, [s.buffers(len(x)) for x in xs], [i32([m] * 2) for m in [90] + [1] * 40], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for j in range(41):
        for s, xs, bs, n, stream in runs:
            with torch.cuda.stream(stream):
                s(xs[j], n[j], len(xs[j]) // 2, bs[j])
                s.advance()
    torch.cuda.synchronize()
    for s, xs, bs, n, _ in runs:
        s.kv_len.copy_(s.length)
        s.check(bs[-1], [1, 1])


def test_a_captured_call_wants_a_workspace():
    cache, table, _ = make_cache([50], 16, 2, 64)
    pages, visible, _ = lists_for([50], table, 16, 2, 3)
    q = torch.randn(1, 4, 64, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with pytest.raises(ValueError, match="workspace"):
        with torch.cuda.graph(graph, stream=side):
            cache.buddy_kv4_attention_pages(q, visible, pages, torch.empty_like(q))


def test_nothing_to_do():
    cache, table, _ = make_cache([50], 16, 2, 64)
    q = torch.empty(0, 4, 64, device="cuda")
    visible, pages = (torch.empty(*s, dtype=torch.int32, device="cuda") for s in ((0,), (0, 2, 4)))
    cache.buddy_kv4_select(q, cache.empty_bounds(), i32([50]), table, pages, visible, i32([0, 0]), 1)
    cache.buddy_kv4_attention_pages(q, visible, pages, q)
    bounds = cache.empty_bounds()
    cache.buddy_kv4_bounds(bounds, i32([50]), table, i32([0, 0]), 5)
    assert not bounds.any()


# ------------------------------------------------------------------ two callers
@pytest.mark.parametrize("tokens,max_new,widths", [(1, 1, (300, 20000)), (400, 1, (3000, 40000)), (12, 3, (600, 8000))])
def test_selections_over_tables_of_two_widths_by_two_threads(tokens, max_new, widths):
    """Neither call's shared memory is taken from the other's: clusters, CTAs of a token, of four."""
    lens = [16 * 20 - 3] * (tokens // max_new)
    calls, checks = [], []
    for n in widths:
        cache, table, bounds, q = make_select(lens, [max_new] * len(lens), 16, (2, 1, 64), torch.bfloat16, seed=n, max_pages=n)
        pages = torch.full((tokens, 1, 7), 55, dtype=torch.int32, device="cuda")
        visible, kv_len, rows = torch.empty(tokens, dtype=torch.int32, device="cuda"), i32(lens), i32(starts_of([max_new] * len(lens)))
        torch.cuda.synchronize()
        calls.append(functools.partial(cache.buddy_kv4_select, q, bounds, kv_len, table, pages, visible, rows, max_new,
                                       stream=torch.cuda.Stream()))
        checks.append((pages, want_pages(q, bounds, table, lens, [max_new] * len(lens), 16, 7, 1, 1, tokens)[0]))
    at_once(*calls)
    for pages, want in checks:
        np.testing.assert_array_equal(pages.cpu().numpy(), want)


# ------------------------------------------------------------------ bad sequences without tokens
@pytest.mark.parametrize("n_new,where", [([1] * 9, 4), ([1] * 400, 399), ([3, 4, 2, 4, 1], 2), ([1, 4, 0, 0, 1], 3),
                                         ([2] * 300, 299), ([2] * 300, 0), ([4] + [0] * 700, 700), ([1], 0), ([1], 1)])
@pytest.mark.parametrize("row", [10, 700])
def test_select_tells_of_bad_sequences_without_tokens(n_new, where, row):
    """They raise the flag as they do in the attention and the bounds; the others' lists are whole."""
    n_new = n_new[:where] + [0] + n_new[where:]
    lens, max_new = [16 * 9 - 1] * len(n_new), max(n_new)
    cache, table, bounds, q = make_select(lens, n_new, 16, (4, 2, 64), torch.bfloat16, seed=where, max_pages=row)
    wp, wv = want_pages(q, bounds, table, lens, n_new, 16, 3, 1, 1, len(q))
    for n, flag in ((-1, BAD_POSITION), (16 * row + 1, BAD_POSITION), (2 ** 31 - 1, BAD_POSITION), (16 * row, 0), (0, 0)):
        lens[where] = n
        pages, visible = (torch.full(s, 55, dtype=torch.int32, device="cuda") for s in ((len(q), 2, 3), (len(q),)))
        fl = flags()
        cache.buddy_kv4_select(q, bounds, i32(lens), table, pages, visible, i32(starts_of(n_new)), max_new, flags=fl)
        np.testing.assert_array_equal(pages.cpu().numpy(), wp)
        np.testing.assert_array_equal(visible.cpu().numpy(), wv)
        assert fl.item() == flag
        if flag:
            fl.zero_()
            cache.buddy_kv4_bounds(cache.empty_bounds(), i32(lens), table, i32(starts_of(n_new)), max_new, fl)
            assert fl.item() == BAD_POSITION


def test_select_tells_of_row_starts_that_do_not_ascend():
    lens = [16 * 9] * 4
    cache, table, bounds, q = make_select(lens, [1] * 4, 16, (4, 2, 64), torch.bfloat16, max_pages=10)
    for rows, max_new in (([0, 4, 1, 3, 4], 4), ([0, 1, 0, 1, 4], 3), ([0, 2, 1, 2, 3], 2), ([0, 1, 2, 4, 3], 2)):
        pages, visible = (torch.full(s, 55, dtype=torch.int32, device="cuda") for s in ((4, 2, 3), (4,)))
        fl = flags()
        cache.buddy_kv4_select(q, bounds, i32(lens), table, pages, visible, i32(rows), max_new, flags=fl)
        assert fl.item() == BAD_POSITION


@pytest.mark.parametrize("row", [12, 600])
@pytest.mark.parametrize("max_new", [1, 2])
@pytest.mark.parametrize("first,last", [(1, 1), (2 ** 31 - 2, 1), (2 ** 29, 1), (2 ** 29, 2 ** 30)])
def test_select_into_the_longest_lists_there_may_be(row, max_new, first, last):
    """Counts over their entries stay right next to 2^31: single tokens, clusters, tokens that share a walk."""
    lens, budget = [16 * 9 - 3], 2 ** 31 - 1
    cache, table, bounds, q = make_select(lens, [1], 16, (2, 1, 64), torch.bfloat16, max_pages=row)
    pages = torch.full((1, 1, budget), 55, dtype=torch.int32, device="cuda")
    visible, fl = torch.empty(1, dtype=torch.int32, device="cuda"), flags()
    cache.buddy_kv4_select(q, bounds, i32(lens), table, pages, visible, i32([0, 1]), max_new, first, last, fl)
    assert pages[0, 0, :9].tolist() == table[0, :9].tolist() and visible.item() == lens[0] and fl.item() == 0
    for part in pages[0, 0, 9:].split(2 ** 28):
        assert torch.all(part == -1)


# ------------------------------------------------------------------ CTAs by sequences
@pytest.mark.parametrize("batch", [31, 255, 256, 257, 700])
@pytest.mark.parametrize("heads,row", [((4, 2, 64), 30), ((3, 1, 128), 30), ((2, 2, 64), 600)])
def test_select_proposed_tokens_of_many_sequences(batch, heads, row):
    """As many sequences as a CTA has threads, fewer and more; of equal lengths, empty and bad ones among
    them, and rows behind the last: over two heads at once, over one, over tables too wide for two."""
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 16 * 25, batch)]
    for i in range(0, batch, 3):
        lens[i] = 16 * 20 + 7
    for i in range(5, batch, 11):
        lens[i] = 0
    n_new = [int(m) for m in rng.integers(2, 6, batch)]       # (more than four: two chunks)
    n_new[batch - 1], pad = 4, 4 * batch                       # (so that most have as many as the longest)
    for most in (4, 5):
        new = [min(m, most) for m in n_new]
        cache, table, bounds, q = make_select(lens, new, 16, heads, torch.bfloat16, seed=batch, pad=pad, max_pages=row)
        check_select(cache, table, bounds, q, lens, new, 6)
        kv, at, T = list(lens), starts_of(new), len(q)
        for i, n in zip((0, 7, batch // 2, batch - 1), (-1, 16 * row + 1, 2 ** 31 - 1, -2 ** 31)):
            kv[i] = n
        wp, wv = want_pages(q, bounds, table, lens, new, 16, 6, 1, 1, T)
        wp[at[-1]:] = 55
        for i in (0, 7, batch // 2, batch - 1):
            wp[at[i]:at[i + 1]], wv[at[i]:at[i + 1]] = 55, -1
        pages, visible = (torch.full(s, 55, dtype=torch.int32, device="cuda") for s in ((T, heads[1], 6), (T,)))
        fl = flags()
        cache.buddy_kv4_select(q, bounds, i32(kv), table, pages, visible, i32(at), most, flags=fl)
        np.testing.assert_array_equal(pages.cpu().numpy(), wp)
        np.testing.assert_array_equal(visible.cpu().numpy(), wv)
        assert fl.item() == BAD_POSITION
