"""The paged 4-bit cache's kernels against the float64 oracle.

Tolerances, before any run:
  norm and rotation, fp32: a dozen roundings of 2^-24 each, and cos / sin rounded
      to fp32: 2^-20 of the pair's length; bf16 outputs add their rounding, 2^-8.
  stored entries: values of v (no arithmetic before them) equal the oracle's; keys
      lie within half a step of the oracle's, plus 2^-17 of the largest of the group
      for its roundings, and their scales within one unit of 7 bits.
  attention: probabilities of 11 bits (2^-11 of the largest value), fp32 statistics
      (2^-12 of it for thousands of terms), rounding of the output (2^-8 bf16). A
      query in fp32 enters with 11 bits: its scores are off by at most 2^-11 of the
      largest sum of |q k|, and so the probabilities, relatively, by twice that.
"""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O

pytestmark = pytest.mark.gpu
THETA, EPS = 1e4, 1e-5
BAD_POSITION, NO_PAGES, BAD_PAGE = 2, 16, 32


def pkg():
    import paper_2606_09514_gb300 as p
    return p


def dev(x, dtype):
    return torch.as_tensor(np.asarray(x), dtype=dtype, device="cuda")


def i32(x):
    return dev(x, torch.int32)


def flags():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ page plan
def make_plan(length, n_new, page, extra_pages=2, spare=0, n_tok=None, head=3, seed=0):
    rng = np.random.default_rng(seed)
    length, n_new = np.asarray(length), np.asarray(n_new)
    held, after = -(-length // page), -(-(length + n_new) // page)
    row = int(after.max(initial=0)) + extra_pages
    ids = rng.permutation(int(after.sum()) + 50)
    table = -np.ones((len(length), row), np.int64)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = ids[at:at + h]
        at += h
    need = int((after - held).sum())
    free = np.concatenate([np.full(head, 10 ** 6), ids[at:at + need], np.full(spare, 10 ** 6)])
    T = int(n_new.sum()) if n_tok is None else n_tok
    B = len(length)
    t = dict(length=i32(length), n_new=i32(n_new), table=i32(table), free=i32(free), head=i32([head]),
             kv_len=i32(np.full(B, -9)), row_start=i32(np.full(B + 1, -9)),
             slot=torch.full((T,), -9, dtype=torch.int64, device="cuda"), pos=i32(np.full(T, -9)), head_out=i32([-9]),
             flags=flags())
    return t, (length, n_new, table, free, head)


def run_plan(t, page):
    pkg().buddy_page_plan(t["length"], t["n_new"], page, t["table"], t["free"], t["head"], t["kv_len"], t["row_start"],
                          t["slot"], t["pos"], t["head_out"], t["flags"])
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in t.items()}


PLANS = {
    "one": ([0], [1], 16), "nothing": ([5, 0], [0, 0], 16), "boundary": ([15, 16, 17, 0, 32], [1, 1, 1, 16, 17], 16),
    "empty-between": ([7, 0, 0, 0, 64], [0, 0, 3, 0, 1], 64), "prompt": ([100], [70000], 128), "page-1": ([3, 0], [2, 4], 1),
}


@pytest.mark.parametrize("name", list(PLANS))
@pytest.mark.parametrize("pad", [0, 7])
def test_plan(name, pad):
    length, n_new, page = PLANS[name]
    t, ref = make_plan(length, n_new, page, spare=3, n_tok=sum(n_new) + pad)
    got = run_plan(t, page)
    check_plan(got, ref, page, pad)
    again = run_plan(t, page)      # the same call again writes the same
    for k in got:
        np.testing.assert_array_equal(got[k], again[k])


def check_plan(got, ref, page, pad=0):
    length, n_new, table, free, head = ref
    table, kv, rows, slot, pos, head = O.page_plan(length, n_new, page, table, free, head)
    assert got["flags"][0] == 0
    np.testing.assert_array_equal(got["table"], table)
    np.testing.assert_array_equal(got["kv_len"], kv)
    np.testing.assert_array_equal(got["row_start"], rows)
    np.testing.assert_array_equal(got["slot"], np.concatenate([slot, -np.ones(pad, int)]))
    np.testing.assert_array_equal(got["pos"], np.concatenate([pos, -np.ones(pad, int)]))
    assert got["head_out"][0] == head


@pytest.mark.parametrize("batch,page", [(2, 32), (33, 16), (255, 64), (257, 64), (1025, 16), (16384, 128)])
def test_plan_batches(batch, page):
    rng = np.random.default_rng(batch)
    length = rng.integers(0, 300, batch) * (rng.random(batch) < 0.8)
    n_new = rng.integers(0, 6, batch)
    t, ref = make_plan(length, n_new, page, seed=batch)
    check_plan(run_plan(t, page), ref, page)


@pytest.mark.parametrize("what,flag", [("pages", NO_PAGES), ("head", NO_PAGES), ("tokens", BAD_POSITION),
                                       ("length", BAD_POSITION), ("new", BAD_POSITION), ("row", BAD_POSITION)])
def test_plan_failure_writes_nothing(what, flag):
    length, n_new, page = [15, 40, 3], [2, 30, 0], 16
    t, _ = make_plan(length, n_new, page, extra_pages=0, n_tok=31 if what == "tokens" else None)
    if what == "pages":
        t["free"] = t["free"][:-1].contiguous()
    if what == "head":
        t["head"].fill_(-1)
    if what == "length":
        t["length"][2] = -1
    if what == "new":
        t["n_new"][2] = -5
    if what == "row":
        t["n_new"][1] += 2 ** 31 - 100
    before = {k: v.cpu().numpy().copy() for k, v in t.items()}
    got = run_plan(t, page)
    assert got["flags"][0] == flag
    for k in got:
        if k != "flags":
            np.testing.assert_array_equal(got[k], before[k])


# ------------------------------------------------------------------ norm and rotation
HEADS = [(4, 2, 64), (5, 1, 64), (9, 3, 64), (32, 8, 128), (7, 7, 128), (1, 1, 128), (6, 2, 128)]


def make_rows(T, heads, dtype, seed=0, gains=True, max_pos=600):
    nq, nkv, hd = heads
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(T, (nq + 2 * nkv) * hd, generator=g, device="cuda").to(dtype)
    q = qkv[:, :nq * hd].unflatten(1, (nq, hd))
    k = qkv[:, nq * hd:(nq + nkv) * hd].unflatten(1, (nkv, hd))
    v = qkv[:, (nq + nkv) * hd:].unflatten(1, (nkv, hd))
    pos = torch.randint(0, max_pos, (T,), generator=g, device="cuda", dtype=torch.int32)
    rope = pkg().buddy_rope_table(max_pos, hd, THETA)
    gain = [torch.rand(hd, generator=g, device="cuda") + 0.5 if gains else None for _ in range(2)]
    return q, k, v, pos, rope, gain


def f64(x):
    return x.double().cpu().numpy()


def check_turned(got, x, gain, pos, dtype, rows=slice(None)):
    want = O.norm_rope(f64(x), None if gain is None else f64(gain), pos.cpu().numpy(), THETA, EPS)[rows]
    h = want.shape[-1] // 2
    pair = np.sqrt(want[..., :h] ** 2 + want[..., h:] ** 2)
    tol = np.concatenate([pair, pair], -1) * 2.0 ** -20 + 1e-30
    if dtype == torch.bfloat16:
        tol = tol + np.abs(want) * 2.0 ** -8
    # angles of the table are those of a double theta^(-2j/hd): the same here
    err = np.abs(f64(got)[rows] - want)
    assert np.all(err <= tol), (err / tol).max()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gains", [True, False])
def test_norm_rope(heads, dtype, gains):
    for T in (1, 3, 130):
        q, k, _, pos, rope, gain = make_rows(T, heads, dtype, seed=T, gains=gains)
        qo, ko = torch.full_like(q.contiguous(), 7), torch.full_like(k.contiguous(), 7)
        fl = flags()
        pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, *gain, EPS, fl)
        check_turned(qo, q, gain[0], pos, dtype)
        check_turned(ko, k, gain[1], pos, dtype)
        assert fl.item() == 0
        # one by one, and in place: the same bits
        q1, k1 = q.clone(), k.clone()
        for t in range(T):
            s = slice(t, t + 1)
            pkg().buddy_qk_norm_rope(q1[s], k1[s], pos[s], rope, q1[s], k1[s], *gain, EPS, fl)
        assert torch.equal(q1, qo) and torch.equal(k1, ko)


def test_norm_of_one_kind_only_and_no_queries():
    q, k, _, pos, rope, gain = make_rows(9, (4, 2, 64), torch.float32)
    qo, ko = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, None, gain[1], EPS)
    check_turned(qo, q, None, pos, torch.float32)
    check_turned(ko, k, gain[1], pos, torch.float32)
    ko2 = torch.empty_like(ko)
    pkg().buddy_qk_norm_rope(None, k, pos, rope, None, ko2, None, gain[1], EPS)
    assert torch.equal(ko, ko2)
    pkg().buddy_qk_norm_rope(q[:0], k[:0], pos[:0], rope, qo[:0], ko[:0], *gain, EPS)


def test_norm_leaves_tokens_out():
    q, k, _, pos, rope, gain = make_rows(5, (4, 2, 64), torch.bfloat16)
    pos[1], pos[3] = -1, 600
    qo, ko = torch.full_like(q.contiguous(), 7), torch.full_like(k.contiguous(), 7)
    fl = flags()
    pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, *gain, EPS, fl)
    assert fl.item() == BAD_POSITION
    for t in (1, 3):
        assert torch.all(qo[t] == 7) and torch.all(ko[t] == 7)
    check_turned(qo, q, gain[0], pos.clamp(0, 599), torch.bfloat16, [0, 2, 4])
    pos[3] = -7
    fl.zero_()
    pkg().buddy_qk_norm_rope(q, k, pos, rope, qo, ko, *gain, EPS, fl)
    assert fl.item() == 0


# ------------------------------------------------------------------ append and read
def read(cache, slot, dtype=torch.float32):
    out = [torch.empty(slot.numel(), cache.n_kv, cache.head_dim, dtype=dtype, device="cuda") for _ in range(2)]
    cache.buddy_kv4_read(slot, *out)
    return out


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("page", [16, 128])
def test_append(heads, dtype, page):
    nq, nkv, hd = heads
    T, n_pages = 77, 9
    q, k, v, pos, rope, gain = make_rows(T, heads, dtype)
    cache = pkg().KV4Cache.empty(n_pages, page, nkv, hd)
    cache.k_pages.fill_(0x5A)
    cache.v_pages.fill_(0x5A)
    slot = torch.randperm(n_pages * page, device="cuda")[:T].contiguous()
    slot[5], slot[6] = -1, -4
    qo, ko = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    fl = flags()
    cache.buddy_kv4_append(q, k, v, pos, slot, rope, qo, *gain, EPS, fl, k_out=ko)
    assert fl.item() == 0
    q2, k2 = torch.empty_like(qo), torch.empty_like(ko)
    pkg().buddy_qk_norm_rope(q, k, pos, rope, q2, k2, *gain, EPS)
    assert torch.equal(qo, q2) and torch.equal(ko, k2)
    kp, vp = (O.entries(x.cpu().numpy(), page, hd).swapaxes(1, 2).reshape(n_pages * page, nkv, hd)
              for x in (cache.k_pages, cache.v_pages))
    s, real = slot.cpu().numpy(), slot.cpu().numpy() >= 0
    codes, scales = O.quantise(f64(v))
    np.testing.assert_array_equal(vp[s[real]], O.values(codes, scales)[real])
    want = O.norm_rope(f64(k), f64(gain[1]), pos.cpu().numpy(), THETA, EPS)[real]
    _, sk = O.quantise(want)
    step = np.repeat(sk, 32, -1)
    big = np.repeat(np.abs(want).reshape(*want.shape[:-1], -1, 32).max(-1), 32, -1)
    assert np.all(np.abs(kp[s[real]] - want) <= step * (0.5 + 7 * 2.0 ** -6) + big * 2.0 ** -17)
    # nothing else was touched
    held = np.ones(n_pages * page, bool)
    held[s[real]] = False
    empty = O.entries(np.full((1, 1, page * (hd // 2 + hd // 16)), 0x5A, np.uint8), page, hd)[0, 0, 0]
    assert np.all(kp[held] == empty) and np.all(vp[held] == empty)
    # read back, each type
    sl = slot.clone()
    sl[~(slot >= 0)] = slot[0]
    kr, vr = read(cache, sl)
    np.testing.assert_array_equal(f64(kr), kp[sl.cpu().numpy()])
    np.testing.assert_array_equal(f64(vr), vp[sl.cpu().numpy()])
    for dt in (torch.float16, torch.bfloat16):
        k1, v1 = read(cache, sl, dt)
        assert torch.equal(k1, kr.to(dt)) and torch.equal(v1, vr.to(dt))


def test_append_special_values():
    hd, nkv, page = 64, 1, 16
    rope = pkg().buddy_rope_table(8, hd, THETA)
    v = torch.zeros(7, nkv, hd, device="cuda")
    v[1, 0, 3] = float("nan")
    v[2, 0, 5], v[2, 0, 6] = float("inf"), 3.0
    v[3] = 2.0 ** -30
    v[4, 0, 0], v[4, 0, 1] = 7 * 2.0 ** -24, -3 * 2.0 ** -24
    v[5, 0, 0] = 1e30
    v[6, 0, 0], v[6, 0, 1], v[6, 0, 2], v[6, 0, 3] = 7.0, 0.5, 1.5, -2.5     # ties to even
    cache = pkg().KV4Cache.empty(2, page, nkv, hd)
    pos, slot = i32(np.zeros(7)), torch.arange(3, 10, device="cuda")
    cache.buddy_kv4_append(None, v, v, pos, slot, rope, None)     # position 0: the rotation is the identity
    kr, vr = read(cache, slot)
    assert torch.equal(torch.nan_to_num(kr, 9e9), torch.nan_to_num(vr, 9e9)) or torch.isnan(kr[2]).any()
    vr = vr.cpu()
    assert torch.all(vr[0] == 0) and torch.all(vr[3] == 0)
    assert torch.all(torch.isnan(vr[1, 0, :32])) and torch.all(vr[1, 0, 32:] == 0)
    assert vr[2, 0, 5] == 6272 and vr[2, 0, 6] == 0
    assert vr[4, 0, 0] == 7 * 2.0 ** -24 and vr[4, 0, 1] == -3 * 2.0 ** -24
    assert vr[5, 0, 0] == 6272
    assert vr[6, 0, :4].tolist() == [7.0, 0.0, 2.0, -2.0]


def test_append_and_read_leave_bad_slots_out():
    q, k, v, pos, rope, gain = make_rows(4, (4, 2, 64), torch.bfloat16)
    cache = pkg().KV4Cache.empty(2, 16, 2, 64)
    slot = dev([0, 32, 5, -1], torch.int64)
    qo = torch.full_like(q.contiguous(), 7)
    fl = flags()
    cache.buddy_kv4_append(q, k, v, pos, slot, rope, qo, *gain, EPS, fl)
    assert fl.item() == BAD_PAGE
    check_turned(qo, q, gain[0], pos, torch.bfloat16)      # the queries of all four are there
    out = [torch.full((4, 2, 64), 7.0, device="cuda") for _ in range(2)]
    fl.zero_()
    cache.buddy_kv4_read(slot, *out, fl)
    assert fl.item() == BAD_PAGE
    for x in out:
        assert torch.all(x[1] == 7) and torch.all(x[3] == 7) and not torch.any(x[0] == 7)


# ------------------------------------------------------------------ attention
def make_cache(kv_len, page, nkv, hd, seed=0, nan_tail=True, first_page=0, n_pages=None):
    """Random pages, a table over them, and each sequence's values in float64."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in kv_len]
    total = sum(need) + 3
    n_pages = n_pages or first_page + total
    ids = first_page + rng.permutation(total)
    row = max(need + [1]) + 1
    table = np.full((len(kv_len), row), -1)
    vals, made = [], []
    for _ in range(2):
        codes = rng.integers(1, 16, (total, nkv, page, hd))
        scales = rng.integers(64, 128, (total, nkv, page, hd // 32)) / 512.0
        made.append((codes, scales))
    at = 0
    for i, n in enumerate(need):
        mine = ids[at:at + n] - first_page
        table[i, :n] = ids[at:at + n]
        at += n
        vals.append([O.values(c[mine], s[mine]).swapaxes(0, 1).reshape(nkv, n * page, hd)[:, :kv_len[i]]
                     for c, s in made])
        if nan_tail and kv_len[i] % page:
            for _, s in made:
                s[mine[-1], :, kv_len[i] % page:] = np.nan
    pages = []
    for c, s in made:
        x = torch.empty(n_pages, nkv, page * (hd // 2 + hd // 16), dtype=torch.uint8, device="cuda")
        x[first_page:first_page + total] = torch.as_tensor(O.blocks(c, s), device="cuda")
        pages.append(x)
    return pkg().KV4Cache(*pages, page), i32(table), vals


def check_attention(cache, table, vals, kv_len, n_new, nq, dtype=torch.bfloat16, out_dtype=torch.bfloat16, scale=0.0,
                    seed=0, amp=1.5, pad=0, ragged=None, strided=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    hd, T = cache.head_dim, sum(n_new) + pad
    q = (amp * torch.randn(T, nq, hd, generator=g, device="cuda")).to(dtype)
    out = torch.full((T, nq, hd), 77.0, dtype=out_dtype, device="cuda")
    if strided:
        q = torch.cat([q, q], 1)[:, :nq]
        out = torch.cat([out, out], 1)[:, nq:]
    starts = np.concatenate([[0], np.cumsum(n_new)])
    rows = None if ragged is False else i32(starts)
    fl = flags()
    for _ in range(2):     # the second call finds the workspace as the first left it
        first = out.clone()
        out.fill_(77.0)
        cache.buddy_kv4_attention(q, i32(kv_len), table, out, rows, max(n_new) if rows is not None else 1, scale, fl)
    assert torch.equal(out, first)
    assert fl.item() == 0
    got, sc = f64(out), scale or 1 / np.sqrt(hd)
    for i, (n, m) in enumerate(zip(kv_len, n_new)):
        if not m:
            continue
        k, v = vals[i]
        qi = f64(q[starts[i]:starts[i] + m])
        want = O.attention(qi, k, v, m, sc)
        top = np.abs(v).max(initial=0.0)
        tol = top * (2.0 ** -11 + 2.0 ** -12) + np.abs(want) * (2.0 ** -8 if out_dtype == torch.bfloat16 else 2.0 ** -22)
        if dtype == torch.float32 and n:
            most = max(np.abs(qi[:, h]).dot(np.abs(k[h // (nq // len(k))]).T).max() for h in range(nq))
            tol = tol + top * 2 * np.expm1(2.0 ** -11 * sc * most)
        err = np.abs(got[starts[i]:starts[i] + m] - want)
        assert np.all(err <= tol), (i, n, m, (err / np.maximum(tol, 1e-30)).max())
    assert np.all(got[starts[-1]:] == 77.0)
    return out


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 511, 1000]


@pytest.mark.parametrize("heads", [(4, 2, 64), (5, 1, 64), (8, 1, 128), (7, 7, 128), (14, 2, 128), (9, 3, 64)])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_attention_single_tokens(heads, page):
    nq, nkv, hd = heads
    cache, table, vals = make_cache(LENGTHS, page, nkv, hd, seed=page)
    check_attention(cache, table, vals, LENGTHS, [1] * len(LENGTHS), nq, ragged=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.0, 0.3])
def test_attention_types_scales_strides(dtype, out_dtype, scale):
    lens = [5, 130, 0, 77]
    cache, table, vals = make_cache(lens, 32, 2, 64)
    for ragged in (False, True):
        check_attention(cache, table, vals, lens, [1] * 4, 6, dtype, out_dtype, scale, ragged=ragged, strided=ragged)
    check_attention(cache, table, vals, lens, [40, 60, 3, 20], 6, dtype, out_dtype, scale, strided=True)


@pytest.mark.parametrize("heads", [(8, 2, 64), (6, 2, 128), (3, 3, 128), (8, 1, 128)])
@pytest.mark.parametrize("n_new", [[2] * 6, [1, 2, 3, 4, 5, 0], [8, 1, 0, 7, 5, 8], [17, 1, 33, 0, 2, 9]])
def test_attention_a_few_tokens(heads, n_new):
    nq, nkv, hd = heads
    lens = [8, 1, 0, 300, 65, 1000]
    cache, table, vals = make_cache(lens, 16, nkv, hd, seed=1)
    check_attention(cache, table, vals, lens, n_new, nq, pad=3)


@pytest.mark.parametrize("heads", [(8, 2, 64), (7, 1, 128), (4, 4, 128), (6, 2, 128)])
@pytest.mark.parametrize("page", [16, 128])
def test_attention_prompts(heads, page):
    """Whole prompts, pieces behind a prefix, single tokens between them, more query
    tokens than positions, and sequences with nothing."""
    nq, nkv, hd = heads
    lens = [129, 700, 41, 0, 350, 20, 256]
    n_new = [129, 300, 1, 5, 0, 70, 128]
    cache, table, vals = make_cache(lens, page, nkv, hd, seed=2)
    check_attention(cache, table, vals, lens, n_new, nq, pad=2)


def test_attention_one_long_sequence():
    for n in (20011, 65536):
        cache, table, vals = make_cache([n], 64, 2, 64, seed=n)
        check_attention(cache, table, vals, [n], [1], 8, ragged=False)
    check_attention(cache, table, vals, [n], [3], 8)
    check_attention(cache, table, vals, [n], [50], 8)


@pytest.mark.parametrize("heads", [(2, 2, 128), (3, 1, 64), (8, 1, 128), (7, 7, 64)])
@pytest.mark.parametrize("lens", [[40001], [9000, 13000], [3000, 20, 6000, 17, 5000]])
def test_attention_streams_of_many_shares(heads, lens):
    """Streams that tens of CTAs share, next to streams that begin and end in the same CTAs:
    few and many rows per join."""
    nq, nkv, hd = heads
    cache, table, vals = make_cache(lens, 64, nkv, hd, seed=len(lens))
    check_attention(cache, table, vals, lens, [1] * len(lens), nq, ragged=False)
    check_attention(cache, table, vals, lens, [2] * len(lens), nq, out_dtype=torch.float32)


def test_attention_many_sequences():
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 90, 700)]
    cache, table, vals = make_cache(lens, 16, 2, 64, seed=3)
    check_attention(cache, table, vals, lens, [1] * 700, 4, ragged=False)
    check_attention(cache, table, vals, lens, [int(x) for x in rng.integers(0, 4, 700)], 4)


def test_attention_peaked_and_flat_scores():
    lens = [900, 33]
    cache, table, vals = make_cache(lens, 64, 2, 128, seed=4)
    check_attention(cache, table, vals, lens, [1, 1], 8, amp=40.0)
    check_attention(cache, table, vals, lens, [1, 1], 8, amp=0.0)
    check_attention(cache, table, vals, lens, [300, 20], 8, amp=40.0)
    check_attention(cache, table, vals, lens, [300, 20], 8, amp=1e-30)


def test_attention_offsets_past_32_bits():
    """Pages at the end of a cache of more than 2^32 bytes."""
    nkv, hd, page = 8, 128, 128
    first = 2 ** 32 // (nkv * page * 72) + 5
    lens = [300, 128]
    cache, table, vals = make_cache(lens, page, nkv, hd, first_page=first)
    assert cache.k_pages.numel() > 2 ** 32
    check_attention(cache, table, vals, lens, [1, 1], 8)
    check_attention(cache, table, vals, lens, [100, 70], 8)
    v = torch.randn(3, nkv, hd, device="cuda")
    slot = torch.arange(3, device="cuda") + (cache.k_pages.shape[0] - 1) * page + 9
    cache.buddy_kv4_append(None, v, v, i32([0, 0, 0]), slot, pkg().buddy_rope_table(4, hd, THETA), None)
    codes, scales = O.quantise(f64(v))
    np.testing.assert_array_equal(f64(read(cache, slot)[1]), O.values(codes, scales))


def test_attention_nan_entries_reach_their_readers_only():
    lens = [40, 40, 200]
    cache, table, vals = make_cache(lens, 16, 1, 64, nan_tail=False)
    page = int(table[1, 0])
    cut = 16 * 32
    cache.v_pages[page, 0, cut:cut + 2] = 0xFF           # position 0 of sequence 1, its first 32 channels
    cache.k_pages[int(table[2, 12]), 0, cut + 4 * 7:] = 0xFF   # keys of sequence 2 from position 199 on
    q = torch.randn(3, 4, 64, device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    cache.buddy_kv4_attention(q, i32(lens), table, out)
    assert torch.isfinite(out[0]).all()
    assert torch.isnan(out[1, :, :32]).all() and torch.isfinite(out[1, :, 32:]).all()
    assert torch.isnan(out[2]).all()
    out2 = torch.empty_like(q)
    cache.buddy_kv4_attention(q, i32([40, 0, 199]), table, out2)
    assert torch.isfinite(out2).all() and torch.all(out2[1] == 0) and torch.equal(out2[0], out[0])
    # queries of a prompt: those behind the bad key see it, the others do not
    q = torch.randn(150, 4, 64, device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    cache.buddy_kv4_attention(q, i32([200]), table[2:], out, i32([0, 150]), 150)
    assert torch.isnan(out[149]).all() and torch.isfinite(out[:149]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [1, 4, 150])
def test_attention_huge_queries_reach_their_own_rows_only(m, dtype):
    """Infinities, NaN and elements beyond a half's range, each in one (token, head).

    A query with one element of 2^17 has scores that are single products, off by two
    roundings of 2^-24 (the factor, the exponent); the other rows as everywhere.
    """
    hd, lens = 64, [210, 170]
    cache, table, vals = make_cache(lens, 16, 1, hd, nan_tail=False)
    q = torch.randn(2 * m, 4, hd, device="cuda").bfloat16().to(dtype)
    q[0, 0], q[m, 1, 5], q[m, 2, 9] = 0.0, float("inf"), float("nan")
    q[0, 0, 3] = 2.0 ** 17
    out = torch.empty_like(q, dtype=torch.float32)
    cache.buddy_kv4_attention(q, i32(lens), table, out, i32([0, m, 2 * m]), m)
    got = f64(out)
    assert not np.isfinite(got[m, 1]).any() and not np.isfinite(got[m, 2]).any()
    for i in range(2):
        k, v = vals[i]
        qi = f64(q[i * m:(i + 1) * m])
        bad = ~np.isfinite(qi).all(-1)
        want = O.attention(np.where(bad[..., None], 0.0, qi), k, v, m, hd ** -0.5)
        top = np.abs(v).max()
        tol = np.full(bad.shape, top * (2.0 ** -11 + 2.0 ** -12))
        if i == 0:
            tol[0, 0] += top * 2 * np.expm1(2 * 2.0 ** -24 * 2.0 ** 17 * np.abs(k[0, :, 3]).max() * hd ** -0.5 * 2)
        err = np.abs(got[i * m:(i + 1) * m] - want).max(-1)
        assert np.all((err <= tol) | bad), (err / tol)[~bad].max()


@pytest.mark.parametrize("n_new", [1, 40])
def test_attention_reports_bad_lengths_and_pages(n_new):
    lens = [70, 70, 70, 70]
    cache, table, vals = make_cache(lens, 16, 2, 64, nan_tail=False)
    T = 4 * n_new
    q = torch.randn(T, 4, 64, device="cuda", dtype=torch.bfloat16)
    rows = i32(np.arange(5) * n_new)
    ok, out, fl = torch.empty_like(q), torch.empty_like(q), flags()
    cache.buddy_kv4_attention(q, i32(lens), table, ok, rows, n_new, flags=fl)
    assert fl.item() == 0
    for bad in (-1, table.shape[1] * 16 + 1):
        out.fill_(77.0)
        cache.buddy_kv4_attention(q, i32([70, bad, 70, 70]), table, out, rows, n_new, flags=fl)
        assert fl.item() == BAD_POSITION
        fl.zero_()
        assert torch.all(out[n_new:2 * n_new] == 77)
        assert torch.equal(out[:n_new], ok[:n_new]) and torch.equal(out[2 * n_new:], ok[2 * n_new:])
    # a page that is not there: its positions do not count
    for bad in (-1, cache.k_pages.shape[0], 2 ** 31 - 1):
        t2 = table.clone()
        t2[2, 1] = bad
        cache.buddy_kv4_attention(q, i32(lens), t2, out, rows, n_new, flags=fl)
        assert fl.item() == BAD_PAGE
        fl.zero_()
        k, v = ([np.delete(x, np.s_[16:32], 1) for x in vals[2]])
        if n_new == 1:
            want = O.attention(f64(q[2:3]), k, v, 1, 0.125)
            assert np.abs(f64(out[2:3]) - want).max() <= np.abs(v).max() * 2.0 ** -10 + np.abs(want).max() * 2.0 ** -8
        assert torch.equal(out[:2 * n_new], ok[:2 * n_new]) and torch.equal(out[3 * n_new:], ok[3 * n_new:])


@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("copies", [1, 40, 700])
def test_attention_without_some_pages(page, copies):
    """Pages that are not there, in every place of a chunk and of a sequence: their positions
    do not count, whoever walks the sequence (one warp, a CTA, many CTAs).  What was in the
    buffers before is NaN in the pages that are there behind the sequences' ends."""
    lens = [5, 33, 250, 300, 47, 1200] * copies if copies < 700 else [5, 33, 250, 40] * copies
    cache, table, vals = make_cache(lens, page, 1, 64, seed=11)
    rng = np.random.default_rng(page)
    lost = []
    t2 = table.clone()
    for i, n in enumerate(lens):
        held = -(-n // page)
        which = {0: [0], 1: [held - 1], 2: range(held)}.get(i % 5, rng.permutation(held)[:rng.integers(0, held + 1)])
        for w in which:
            t2[i, int(w)] = -1 if w % 2 else cache.k_pages.shape[0] + 5
        lost.append(np.isin(np.arange(n) // page, np.asarray(list(which), int)))
    q = torch.randn(len(lens), 3, 64, device="cuda").bfloat16()
    out, fl = torch.full((len(lens), 3, 64), 77.0, device="cuda"), flags()
    cache.buddy_kv4_attention(q, i32(lens), t2, out, flags=fl)
    assert fl.item() == BAD_PAGE
    got = f64(out)
    for i, gone in enumerate(lost[:200]):
        k, v = (x[:, ~gone] for x in vals[i])
        want = O.attention(f64(q[i:i + 1]), k, v, 1, 0.125) if (~gone).any() else np.zeros((1, 3, 64))
        tol = np.abs(v).max(initial=0.0) * (2.0 ** -11 + 2.0 ** -12) + 2.0 ** -22 * np.abs(want)
        assert np.all(np.abs(got[i:i + 1] - want) <= tol), (i, lens[i])


@pytest.mark.parametrize("rows", [[0, 1, 3, 2, 4], [-1, 1, 2, 3, 4], [0, 1, 2, 3, 9], [0, 1, 4, 4, 4]])
def test_attention_with_bad_row_starts(rows):
    """More rows than max_new, descending, or outside q: reported, nothing outside is touched."""
    lens = [70, 70, 70, 70]
    cache, table, _ = make_cache(lens, 16, 2, 64)
    q = torch.randn(4, 4, 64, device="cuda", dtype=torch.bfloat16)
    buf = torch.full((12, 4, 64), 77.0, device="cuda", dtype=torch.bfloat16)
    fl = flags()
    cache.buddy_kv4_attention(q, i32(lens), table, buf[4:8], i32(rows), 2, flags=fl)
    assert fl.item() == BAD_POSITION
    assert torch.all(buf[:4] == 77) and torch.all(buf[8:] == 77)


def test_attention_shares_a_workspace_between_shapes_and_streams():
    a = make_cache([500, 3, 80], 16, 2, 64, seed=7)
    b = make_cache([2000], 64, 4, 128, seed=8)
    ws = torch.zeros(max(a[0].workspace_bytes(8, 64), b[0].workspace_bytes(8, 64)), dtype=torch.uint8, device="cuda")
    a[0].workspace = b[0].workspace = ws
    side = torch.cuda.Stream()
    for n_new in (1, 3, 60):
        check_attention(*a, [500, 3, 80], [n_new, 1, n_new], 8)
        check_attention(*b, [2000], [n_new], 8)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            check_attention(*a, [500, 3, 80], [n_new, 1, n_new], 8)
        side.synchronize()


def test_calls_refuse_wrong_tensors():
    """A wrong type, device, shape, stride or size of any tensor: an error that names it, and
    nothing written."""
    P, T, nq, nkv, hd, page = pkg(), 6, 4, 2, 64, 16
    cache = P.KV4Cache.empty(4, page, nkv, hd)
    co, si = P.buddy_rope_table(8, hd, THETA)
    x = torch.randn(T, nq + nkv, hd, device="cuda").bfloat16()
    q, k, v, q_out = x[:, :nq], x[:, nq:], x[:, nq:], torch.full((T, nq, hd), 7.0, device="cuda").bfloat16()
    pos, slot = i32([0] * T), torch.arange(T, device="cuda")
    gain = torch.ones(hd, device="cuda")
    good = dict(q=q, k=k, v=v, pos=pos, slot=slot, rope=(co, si), q_out=q_out, q_gain=gain, k_gain=gain, flags=flags())

    def check(call, good, bad, untouched):
        for name, value in bad:
            before = [t.clone() for t in untouched]
            with pytest.raises((ValueError, TypeError)) as e:
                call(**{**good, name: value})
            assert any(w in str(e.value) for w in (name, "cos", "sin")), (name, e.value)
            assert all(torch.equal(a, b) for a, b in zip(before, untouched)), name

    pages = [cache.k_pages, cache.v_pages, q_out]
    check(cache.buddy_kv4_append, good, [
        ("q", q.float()), ("q", q.cpu()), ("q", q[:-1]), ("q", q[0]), ("q", q.transpose(1, 2).contiguous().transpose(1, 2)),
        ("k", k.half()[0]), ("k", x[:, ::3]), ("k", None), ("v", v[:, :1]), ("v", v.float()), ("v", 3), ("pos", pos.long()),
        ("pos", pos[:-1]), ("pos", torch.zeros(2 * T, device="cuda", dtype=torch.int32)[::2]), ("slot", slot.int()),
        ("slot", slot[:-1]), ("rope", (co.double(), si)), ("rope", (co, si[:-1])), ("q_out", None), ("q_out", q_out[:, :-1]),
        ("q_gain", gain[:-1]), ("k_gain", gain.bfloat16()), ("flags", flags().cpu())], pages)
    out = torch.empty(T, nkv, hd, device="cuda")
    check(cache.buddy_kv4_read, dict(slot=slot, k_out=out, v_out=out, flags=None), [
        ("slot", slot.int()), ("k_out", out.double()), ("k_out", out[:-1]), ("v_out", out.half()), ("flags", 1)], [out])
    att = dict(q=q, kv_len=i32([3] * T), table=i32([[0]] * T), out=q_out, row_start=i32(range(T + 1)), flags=None)
    check(cache.buddy_kv4_attention, att, [
        ("q", q[:, :, :32]), ("q", q[0]), ("kv_len", i32([3] * T).long()), ("table", i32([0] * T)), ("table", i32([[0]] * 2)),
        ("out", q_out[:-1]), ("out", q_out.cpu()), ("row_start", i32(range(T))), ("workspace", flags())], [q_out])
    t, _ = make_plan([15, 3], [2, 30], page)
    plan = dict(length=t["length"], n_new=t["n_new"], page_size=page, table=t["table"], free_pages=t["free"],
                free_head=t["head"], kv_len=t["kv_len"], row_start=t["row_start"], slot=t["slot"], pos=t["pos"],
                free_head_out=t["head_out"], flags=t["flags"])
    check(P.buddy_page_plan, plan, [
        ("length", t["length"].long()), ("length", [1, 2]), ("n_new", t["n_new"][:1]), ("table", t["table"][0]),
        ("table", t["table"][:, ::2]), ("free_pages", t["free"].long()), ("free_head", t["head"].cpu()),
        ("kv_len", t["kv_len"][:1]), ("row_start", t["kv_len"]), ("slot", t["pos"]), ("pos", t["pos"][:-1]),
        ("free_head_out", t["head_out"].float())], [t["table"], t["slot"], t["pos"], t["kv_len"]])
    with pytest.raises(OverflowError):
        P.buddy_page_plan(**{**plan, "page_size": 2 ** 40})
    with pytest.raises(P.BuddyError):
        P.buddy_page_plan(**{**plan, "page_size": 48})
    with pytest.raises(P.BuddyError):          # a workspace that is too small
        cache.buddy_kv4_attention(**{**att, "workspace": torch.zeros(4096, dtype=torch.uint8, device="cuda")})
    side = torch.cuda.Stream()
    cache.buddy_kv4_append(**good, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert good["flags"].item() == 0 and torch.isfinite(q_out).all()


@pytest.mark.parametrize("m", [1, 3, 40])
def test_calls_in_a_row_wait_for_each_other(m):
    """Launches may overlap their predecessors' ends: a chain of calls with ordinary kernels
    between them, enqueued at once, gives what it gives with the host waiting after each."""
    nq, nkv, hd, page, B = 8, 2, 64, 16, 6
    rope = pkg().buddy_rope_table(4096, hd, THETA)
    g = torch.Generator(device="cuda").manual_seed(3)
    src = torch.randn(12, B * m, nq + 2 * nkv, hd, generator=g, device="cuda").bfloat16()
    big = torch.randn(2048, 2048, device="cuda", generator=g)

    def chain(wait):
        cache = pkg().KV4Cache.empty(B * 64, page, nkv, hd)
        table = torch.full((B, 64), -1, dtype=torch.int32, device="cuda")
        free, head = torch.randperm(B * 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).int(), i32([0])
        length, n_new, kv, rows, head2 = i32([0] * B), i32([m] * B), i32([0] * B), i32([0] * (B + 1)), i32([0])
        slot, pos = torch.zeros(B * m, dtype=torch.int64, device="cuda"), i32([0] * (B * m))
        x, q, k, fl, got = torch.empty_like(src[0]), torch.empty_like(src[0][:, :nq]), None, flags(), []
        out = torch.empty_like(q)
        kr = torch.empty(B * m, nkv, hd, dtype=torch.float32, device="cuda")
        for i in range(len(src)):
            (big @ big).sum()                       # something that takes a while
            steps = [
                lambda: x.copy_(src[i]),
                lambda: pkg().buddy_page_plan(length, n_new, page, table, free, head, kv, rows, slot, pos, head2, fl),
                lambda: cache.buddy_kv4_append(x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], pos, slot, rope, q, flags=fl),
                lambda: x.zero_(),
                lambda: cache.buddy_kv4_attention(q, kv, table, out, rows, m, flags=fl),
                lambda: cache.buddy_kv4_read(slot, kr, None, fl),
                lambda: pkg().buddy_qk_norm_rope(None, kr, pos, rope, None, kr, flags=fl),
                lambda: q.zero_(),
                lambda: (got.append(out.clone()), got.append(kr.clone())),
                lambda: (length.copy_(kv), head.copy_(head2), slot.fill_(-1), out.zero_()),
            ]
            for step in steps:
                step()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert fl.item() == 0
        return got

    for a, b in zip(chain(False), chain(True)):
        assert torch.equal(a, b) and torch.isfinite(a).all()


def test_step_in_a_graph():
    """Plan, append and attention captured once, replayed as the sequences grow."""
    nq, nkv, hd, page, B = 6, 2, 64, 16, 5
    rng = np.random.default_rng(11)
    length = np.array([0, 15, 16, 30, 47])
    t, _ = make_plan(length, [1] * B, page, extra_pages=2)
    t["free"] = i32(100 + rng.permutation(40))
    t["head"].zero_()
    table0 = t["table"].clone()
    cache = pkg().KV4Cache.empty(140, page, nkv, hd)
    rope = pkg().buddy_rope_table(200, hd, THETA)
    q, k, v = (torch.empty(B, h, hd, device="cuda", dtype=torch.bfloat16) for h in (nq, nkv, nkv))
    qo, out = torch.empty_like(q), torch.empty_like(q)
    cache.workspace = torch.zeros(cache.workspace_bytes(nq), dtype=torch.uint8, device="cuda")

    def step():
        pkg().buddy_page_plan(t["length"], t["n_new"], page, t["table"], t["free"], t["head"], t["kv_len"],
                              t["row_start"], t["slot"], t["pos"], t["head_out"], t["flags"])
        cache.buddy_kv4_append(q, k, v, t["pos"], t["slot"], rope, qo, flags=t["flags"])
        cache.buddy_kv4_attention(qo, t["kv_len"], t["table"], out, t["row_start"], 1, flags=t["flags"])

    def advance():
        t["length"].copy_(t["kv_len"])
        t["head"].copy_(t["head_out"])

    held = [[np.zeros((nkv, 0, hd))] * 2 for _ in range(B)]
    for i, n in enumerate(length):   # what the sequences hold before
        if n:
            x = torch.randn(int(n), nkv, hd, device="cuda").bfloat16()
            slot = table0[i].long().repeat_interleave(page) * page + torch.arange(table0.shape[1] * page, device="cuda") % page
            cache.buddy_kv4_append(None, x, x, i32(np.zeros(n)), slot[:n].contiguous(), rope, None)
            held[i] = [f64(y).swapaxes(0, 1) for y in read(cache, slot[:n].contiguous())]
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        step()
    for n in range(20):
        for x in (q, k, v):
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert t["flags"].item() == 0
        new = [f64(y) for y in read(cache, t["slot"])]
        for i in range(B):
            held[i] = [np.concatenate([h, x[i][:, None]], 1) for h, x in zip(held[i], new)]
            want = O.attention(f64(qo[i:i + 1]), *held[i], 1, 1 / np.sqrt(hd))
            tol = np.abs(held[i][1]).max() * (2.0 ** -11 + 2.0 ** -12) + np.abs(want) * 2.0 ** -8
            assert np.all(np.abs(f64(out[i:i + 1]) - want) <= tol), (n, i)
        advance()
