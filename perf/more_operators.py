"""Measured cases of what a serving program calls for long contexts over the paged 4-bit
cache: rotation by several position axes, and attention over the pages that a cheap score
selects for each query, through the package's public entry points.

A case is a dict of plain values:
  op       "axes" (buddy_qk_norm_rope with axes), "append" (buddy_kv4_append with axes, and
           buddy_kv4_read of what it stored), "bounds" (buddy_kv4_bounds), "select"
           (buddy_kv4_select) or "pages" (buddy_kv4_attention_pages)
  tokens   tokens of the call (axes, append)
  sections frequencies of each position axis, "16 24 24"; round: taken in turn, not in runs
  batch    sequences (bounds, select, pages)
  lo, hi   positions that a sequence holds before the call, spread over [lo, hi] (over their
           logarithm); every 16th sequence holds nothing
  new_lo, new_hi   new tokens per sequence
  budget   pages of a query; the first and the last page are always among them
  heads, kv_heads, dim   head layout
  page     positions per page
  dtype    "f32" or "bf16": type of q, k, v and the outputs
  gains    queries and keys are normalised for each head before the rotation
  spread   seed of the lengths: they belong to the case, the values to the seed
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

EPS = 1e-6
THETA = 1e6
GROUP = 32          # channels that share a scale
NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)   # channel of a word of eight -> nibble that holds it
ANGLES = 8320       # rows of the rotary tables

# (query heads, KV heads, head dim): grouped heads of 128, as many KV heads as
# query heads, odd groups, heads of 64
HEADS = ((32, 8, 128), (28, 4, 128), (40, 40, 128), (6, 2, 128), (9, 3, 64), (4, 4, 64), (5, 1, 64))
# halves of a head's frequencies over time, height and width, or height and width
SECTIONS = {128: ("16 24 24", "24 20 20", "32 32", "10 20 14 20"), 64: ("8 12 12", "12 10 10", "16 16", "5 9 9 9")}


# --------------------------------------------------------------------------- cases
def _rows(name, op, tokens, heads, dtype, gains, sections, turns, page=64):
    c = {"op": op, "tokens": tokens, "heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype,
         "gains": gains, "sections": sections, "round": turns, "page": page}
    return {**c, "name": name} if name else c


def _pages(name, op, batch, lo, hi, new_lo, new_hi, heads, dtype, page, budget, spread):
    c = {"op": op, "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "heads": heads[0],
         "kv_heads": heads[1], "dim": heads[2], "dtype": dtype, "page": page, "budget": budget, "spread": spread}
    return {**c, "name": name} if name else c


def listed():
    return [
        # one user's next token
        _rows("axes-1", "axes", 1, (32, 8, 128), "bf16", True, "16 24 24", False),
        # the patches of some images and the text around them
        _rows("axes-7901", "axes", 7901, (32, 8, 128), "bf16", True, "16 24 24", False),
        # a decode batch of a model in 32 bits whose axes take the frequencies in turn
        _rows("append-f32-250", "append", 250, (28, 4, 128), "f32", True, "24 20 20", True, 64),
        # a video's prompt, without the norms
        _rows("append-5003", "append", 5003, (28, 4, 128), "bf16", False, "16 24 24", False, 32),
        # a full server's next token: the page that each sequence writes to
        _pages("bounds-250", "bounds", 250, 512, 8192, 1, 1, (28, 4, 128), "bf16", 64, 32, 1),
        # all pages of a long document that has come from elsewhere
        _pages("bounds-120001", "bounds", 1, 0, 0, 120001, 120001, (32, 8, 128), "bf16", 64, 64, 2),
        # one user's next token over a long document
        _pages("select-1", "select", 1, 120001, 120001, 1, 1, (32, 8, 128), "bf16", 64, 64, 3),
        # a full server, requests of all ages, idle slots among them
        _pages("select-250", "select", 250, 512, 8192, 1, 1, (28, 4, 128), "bf16", 64, 32, 4),
        # several proposed tokens of each request, small pages, a KV head for each query head
        _pages("select-31", "select", 31, 400, 12000, 1, 5, (40, 40, 128), "bf16", 16, 64, 5),
        # the same calls' attention
        _pages("pages-1", "pages", 1, 120001, 120001, 1, 1, (32, 8, 128), "bf16", 64, 64, 6),
        _pages("pages-250", "pages", 250, 512, 8192, 1, 1, (28, 4, 128), "bf16", 64, 32, 7),
        _pages("pages-31", "pages", 31, 100, 4096, 1, 5, (40, 40, 128), "bf16", 16, 64, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(("axes", "append", "bounds", "select", "select", "pages", "pages"))
    heads, page, dtype = rng.choice(HEADS), rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "bf16", "f32"))
    spread = rng.randrange(1 << 20)
    if op in ("axes", "append"):
        # a layout of 40 + 80 heads moves four times what 28 + 8 do
        t = _log(rng, 1, (4000 if op == "append" else 7500) // (2 if dtype == "f32" else 1))
        return _rows(None, op, max(1, t * 8 // max(8, heads[1])), heads, dtype, rng.random() < 0.7,
                     rng.choice(SECTIONS[heads[2]]), rng.random() < 0.5, page)
    if op == "bounds":
        # (position, KV head) pairs within what bounds-120001 has
        pairs = 960_000 // heads[1]
        batch = _log(rng, 1, min(250, pairs // 128))
        new = rng.choice((1, _log(rng, 1, max(1, pairs // batch - 128))))
        return _pages(None, op, batch, 1, _log(rng, 1, 8192), max(1, new // 8), new, heads, dtype, page, 1, spread)
    # (token or sequence, KV head, page) triples within what select-31 has; (token, KV head,
    # position) ones within what pages-250 and pages-31 have
    kind = rng.choice(("decode", "decode", "verify", "prompts"))
    batch = _log(rng, 1, {"decode": 250, "verify": 40, "prompts": 4}[kind])
    new = {"decode": 1, "verify": rng.randint(2, 8), "prompts": _log(rng, 20, 400)}[kind]
    rows = batch * new * heads[1]
    hi = _log(rng, 1, max(2, min(100000, (200_000 if new == 1 else 900_000) // rows * page)))
    budget = _log(rng, 2, max(2, min(128, 1_800_000 // rows // page)))
    return _pages(None, op, batch, max(1, hi // 16), hi, max(1, new // 4) if kind == "prompts" else 1, new, heads, dtype,
                  page, budget, spread)


def _lengths(case):
    """Positions of each sequence, the call's new ones among them (idle slots: 0), and its new tokens."""
    rng = random.Random("lengths %d" % case["spread"])
    have, new = [], []
    for i in range(case["batch"]):
        n = 0 if case["hi"] == 0 else _log(rng, max(1, case["lo"]), case["hi"])
        m = rng.randint(case["new_lo"], case["new_hi"])
        if i % 4 == 3:        # a request that decodes next to the others' longer pieces
            m = case["new_lo"]
        have.append(0 if i % 16 == 15 else n + m)
        new.append(m)
    if case["batch"] > 1:     # the longest piece there is
        have[0] += case["new_hi"] - new[0]
        new[0] = case["new_hi"]
    return have, new


def _ceil(n, page):
    return -(-n // page)


def _axis_of(case):
    """The axis of each frequency."""
    counts = [int(s) for s in case["sections"].split()]
    if not case["round"]:
        return [a for a, n in enumerate(counts) for _ in range(n)]
    out = []
    for r in range(max(counts)):
        out += [a for a, n in enumerate(counts) if n > r]
    return out


def work(case):
    op = case["op"]
    nq, nkv, hd = case["heads"], case["kv_heads"], case["dim"]
    e = 4 if case["dtype"] == "f32" else 2
    entry = hd // 2 + hd // 16
    if op in ("axes", "append"):
        t, rotated = case["tokens"], nq + nkv
        b = t * (rotated * hd * e + hd * 4 + 4 * len(case["sections"].split()))   # q, k, cos and sin, positions
        if op == "axes":
            return {"bytes": b + t * rotated * hd * e, "flops": t * rotated * hd * 10}
        b += t * (nkv * hd * e + nq * hd * e + 8 + 2 * nkv * entry)    # v, q's output, slots, the entries stored
        b += t * (8 + 2 * nkv * entry + 2 * nkv * hd * 2)              # the entries read back, and their values
        return {"bytes": b, "flops": t * (rotated * hd * 10 + 2 * nkv * hd * 4)}
    have, new = _lengths(case)
    P, k, first = case["page"], case["budget"], [max(0, h - n) for h, n in zip(have, new)]
    if op == "bounds":
        pages = [_ceil(h, P) - f // P if h else 0 for h, f in zip(have, first)]
        read = [h - f // P * P if h else 0 for h, f in zip(have, first)]
        return {"bytes": nkv * (sum(read) * entry + sum(pages) * 4 * hd) + 4 * sum(pages) + 8 * case["batch"],
                "flops": 2 * nkv * hd * sum(read)}
    own_pages = [[p // P + 1 for p in range(f, h)] for f, h in zip(first, have)]       # of each token
    if op == "select":
        # the bounds of each sequence's pages once; nothing where all pages are taken
        seen = [max([n - 2 for n in pages if n > k] + [0]) for pages in own_pages]
        scored = sum(n - 2 for pages in own_pages for n in pages if n > k)
        return {"bytes": sum(seen) * nkv * 4 * hd + sum(max(n + [0]) for n in own_pages) * 4 + 8 * case["batch"] +
                sum(new) * (nq * hd * e + nkv * k * 4 + 4),
                "flops": 4 * nkv * hd * scored}
    vis = [[(min(n, k) - 1) * P + p % P + 1 for n, p in zip(pages, range(f, h))]
           for pages, f, h in zip(own_pages, first, have)]
    return {"bytes": sum(min(sum(v), h) for v, h in zip(vis, have)) * nkv * 2 * entry + sum(new) * (2 * nq * hd * e + nkv * k * 4 + 4),
            "flops": 4 * nq * hd * sum(sum(v) for v in vis)}


# --------------------------------------------------------------------------- inputs
def _rope(rows, hd, dev):
    a = torch.arange(rows, device=dev, dtype=torch.float64)[:, None] * \
        THETA ** (-2.0 * torch.arange(hd // 2, device=dev, dtype=torch.float64) / hd)
    return a.cos().float(), a.sin().float()


def _random_pages(n_pages, nkv, page, hd, g, dev):
    """Pages as a program finds them after other requests: codes and scales
    everywhere, in plain byte arithmetic, a part of the pages at a time."""
    out = torch.empty(n_pages, nkv, page * (hd // 2 + hd // 16), dtype=torch.uint8, device=dev)
    for a in range(0, n_pages, 4096):
        part = out[a:a + 4096]
        n = part.shape[0]
        x = torch.randn(n, nkv, page * hd // 2, 2, generator=g, device=dev, dtype=torch.float16)
        c = (x.mul_(2.9).round_().clamp_(-7, 7) + 8).to(torch.uint8)
        part[..., :page * hd // 2] = c[..., 0] + 16 * c[..., 1]
        # seven significant bits around 2.3 / 7
        s = torch.randint(64, 128, (n, nkv, page * hd // 32), generator=g, device=dev).to(torch.float16) / 256.0
        part[..., page * hd // 2:] = s.view(torch.uint8)
    return out


def _positions(tokens, axes, g, dev):
    """Position axes of text (all alike) and, of four tokens in five, of image patches: the
    first axis stands, the others run over the patch grid."""
    base = torch.randint(0, ANGLES - 64, (1, tokens), generator=g, device=dev)
    grid = torch.randint(0, 64, (axes, tokens), generator=g, device=dev)
    grid[0] = 0
    text = torch.rand(1, tokens, generator=g, device=dev) < 0.2
    return (base + torch.where(text, torch.zeros_like(grid), grid)).to(torch.int32).contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    op = case["op"]
    st = {"case": case, "flags": torch.zeros(1, dtype=torch.int32, device=dev)}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    nq, nkv, hd, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    if op in ("axes", "append"):
        t = case["tokens"]
        # one projection's output: queries, keys and values of a token side by side;
        # some channels of the keys are larger than the others
        qkv = torch.randn(t, (nq + 2 * nkv) * hd, generator=g, device=dev)
        qkv[:, nq * hd:(nq + nkv) * hd] *= torch.exp(0.4 * torch.randn(nkv * hd, generator=g, device=dev))
        qkv = qkv.to(dt)
        st.update(q=qkv[:, :nq * hd].unflatten(1, (nq, hd)), k=qkv[:, nq * hd:(nq + nkv) * hd].unflatten(1, (nkv, hd)),
                  v=qkv[:, (nq + nkv) * hd:].unflatten(1, (nkv, hd)), rope=_rope(ANGLES, hd, dev),
                  pos=_positions(t, len(case["sections"].split()), g, dev),
                  axis=torch.tensor(_axis_of(case), device=dev),
                  q_gain=None, k_gain=None, q_out=torch.empty(t, nq, hd, dtype=dt, device=dev))
        if case["gains"]:
            st["q_gain"] = torch.rand(hd, generator=g, device=dev) + 0.5
            st["k_gain"] = torch.rand(hd, generator=g, device=dev) + 0.5
        if op == "axes":
            st["k_out"] = torch.empty(t, nkv, hd, dtype=dt, device=dev)
            return st
        # up to 256 tokens: one per request, each in a page of its own; above: prompts,
        # position by position through pages that lie anywhere
        n_pages = (t if t <= 256 else _ceil(t, page)) + 20
        st["k_pages"], st["v_pages"] = (_random_pages(n_pages, nkv, page, hd, g, dev) for _ in range(2))
        ids = torch.randperm(n_pages, generator=g, device=dev)
        if t <= 256:
            st["slot"] = ids[:t] * page + torch.randint(0, page, (t,), generator=g, device=dev)
        else:
            st["slot"] = (ids[:, None] * page + torch.arange(page, device=dev)).reshape(-1)[:t].contiguous()
        st["k_read"], st["v_read"] = (torch.empty(t, nkv, hd, dtype=torch.float16, device=dev) for _ in range(2))
        return st
    have, new = _lengths(case)
    row = max(1, max(_ceil(n, page) for n in have)) + 1
    need = sum(_ceil(n, page) for n in have)
    n_pages = need + 10
    table = torch.full((case["batch"], row), -1, dtype=torch.int32, device=dev)
    used = torch.arange(row, device=dev)[None] < i32([_ceil(n, page) for n in have])[:, None]
    table[used] = torch.randperm(n_pages, generator=g, device=dev)[:need].to(torch.int32)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    T, k = starts[-1], case["budget"]
    st.update(table=table, kv_len=i32(have), row_start=i32(starts) if case["new_hi"] > 1 else None, max_new=max(new))
    if op == "select":
        # what lies in the pages themselves is not looked at
        st["k_pages"], st["v_pages"] = (torch.zeros(n_pages, nkv, page * (hd // 2 + hd // 16), dtype=torch.uint8, device=dev)
                                        for _ in range(2))
        mid = torch.randn(n_pages, nkv, 1, hd, generator=g, device=dev)
        wide = 1.5 + torch.rand(n_pages, nkv, 1, hd, generator=g, device=dev)
        st["bounds"] = torch.cat([mid - wide, mid + wide], 2).half()
    else:
        st["k_pages"], st["v_pages"] = (_random_pages(n_pages, nkv, page, hd, g, dev) for _ in range(2))
        # what no request has written yet is what the memory held: NaN scales here, behind the
        # last position of each sequence
        for i, n in enumerate(have):
            if n % page:
                p = int(table[i, n // page])
                for pages in (st["k_pages"], st["v_pages"]):
                    pages[p, :, page * hd // 2:].unflatten(1, (page, hd // 16))[:, n % page:] = 0xFF
    if op == "bounds":
        # the pages' bounds of before the call
        st["bounds"] = torch.randn(n_pages, nkv, 2, hd, generator=g, device=dev).half()
        return st
    st["q"] = (2 * torch.randn(T, nq, hd, generator=g, device=dev)).to(dt)
    st["pages"], st["visible"] = torch.empty(T, nkv, k, dtype=torch.int32, device=dev), torch.empty(T, dtype=torch.int32, device=dev)
    if op == "pages":
        # lists as a selection leaves them: first and last page, others anywhere between
        seq = torch.repeat_interleave(torch.arange(case["batch"], device=dev), torch.tensor(new, device=dev))
        pos = (st["kv_len"] - i32(new))[seq] + torch.arange(T, device=dev) - torch.tensor(starts, device=dev)[seq]
        held = torch.where(pos >= 0, pos // page + 1, 0)
        st["pages"], st["visible"] = _lists(torch.rand(T, nkv, row, generator=g, device=dev), held, pos, table[seq], k, page)
        st["out"] = torch.empty(T, nq, hd, dtype=dt, device=dev)
    return st


def _lists(score, held, pos, table, k, page):
    """Each row's best `k` of its pages, the first and the last among them, in their order, -1
    behind them, and the positions that they hold. score [tokens, heads, pages]; held, pos
    [tokens]: pages and last position; table [tokens, pages]."""
    T, H, N = score.shape
    j = torch.arange(N, device=score.device)
    # a place in the order: 0 the pages that are always in, 1 by score, 2 those that are not there
    last = (held - 1)[:, None]
    kind = torch.where(j[None] > last, 2, torch.where((j[None] == 0) | (j[None] == last), 0, 1))[:, None].expand(T, H, N)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    order = torch.gather(order, -1, torch.sort(torch.gather(kind, -1, order), dim=-1, stable=True).indices)
    best = order[..., :k]
    count = held.clamp(max=k)
    there = torch.arange(best.shape[-1], device=score.device) < count[:, None, None]
    best = torch.sort(torch.where(there, best, N), dim=-1).values
    ids = torch.gather(table[:, None].expand(T, H, N), -1, best.clamp(max=N - 1))
    pages = torch.full((T, H, k), -1, dtype=torch.int32, device=score.device)
    pages[..., :best.shape[-1]] = torch.where(there, ids, -1)
    return pages, torch.where(held > 0, (count - 1) * page + pos % page + 1, 0).int()


# --------------------------------------------------------------------------- plain form
def _halve(y):
    """Sum over the last axis: the upper half onto the lower, until one is left."""
    n = y.shape[-1]
    return y[..., 0] if n == 1 else _halve(y[..., :n // 2] + y[..., n // 2:])


def _eights(y):
    """Sum over the last axis in the operators' order: eight neighbours, then the eights."""
    return _halve(_halve(y.unflatten(-1, (-1, 8))))


def _turned(x, gain, pos, axis, rope):
    """Norm of each head (where there are gains) and rotation, in 32 bits."""
    x = x.float()
    if gain is not None:
        # the order of the sum is a part of the operator's definition
        x = x * (1.0 / torch.sqrt(_eights(x * x) * (1.0 / x.shape[-1]) + EPS))[..., None] * gain
    at = pos.long()[axis].t()                                                  # [tokens, frequencies]
    c, s = (torch.gather(t, 0, at)[:, None] for t in rope)
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _stored(x):
    """The values that the 4-bit cache holds for x."""
    grp = x.float().unflatten(-1, (-1, GROUP))
    s = grp.abs().amax(-1, keepdim=True) / torch.full((), 7.0, device=x.device)
    m, e = torch.frexp(s)
    s = torch.ldexp(torch.round(m * 128.0), e - 7).clamp(max=896.0).half().float()
    n = torch.where(s > 0, torch.round(grp / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(grp))
    return (n.clamp(-7, 7) * s).flatten(-2)


def _held(blk, page, hd):
    """The values of blocks [..., bytes]: [..., positions, dim] in 32 bits."""
    codes, scales = blk[..., :page * hd // 2], blk[..., page * hd // 2:].contiguous().view(torch.float16)
    nib = torch.stack([codes & 15, codes >> 4], -1).unflatten(-2, (page, hd // 8, 4)).flatten(-2)
    val = nib[..., list(NIBBLE)].flatten(-2).unflatten(-1, (hd // GROUP, GROUP)).float() - 8.0
    return (val * scales.unflatten(-1, (page, hd // GROUP))[..., None].float()).flatten(-2)


def _tokens(st):
    """Of each query token: its sequence and its position."""
    case, kv_len, dev = st["case"], st["kv_len"].long(), st["kv_len"].device
    start = torch.arange(case["batch"] + 1, device=dev) if st["row_start"] is None else st["row_start"].long()
    t = torch.arange(st["q"].shape[0], device=dev)
    seq = (t[:, None] >= start[None, 1:]).sum(1)
    return seq, (kv_len - (start[1:] - start[:-1]))[seq] + t - start[seq]


def _plain_bounds(st):
    case, table = st["case"], st["table"].long()
    P, hd, kv_len, dev = case["page"], case["dim"], st["kv_len"].long(), st["table"].device
    start = torch.arange(case["batch"] + 1, device=dev) if st["row_start"] is None else st["row_start"].long()
    j = torch.arange(table.shape[1], device=dev)[None]
    since = (kv_len - (start[1:] - start[:-1])).clamp(min=0)
    hit = (j >= (since // P)[:, None]) & (j * P < kv_len[:, None])
    seq, col = torch.nonzero(hit, as_tuple=True)
    ids = table[hit]
    K = _held(st["k_pages"][ids], P, hd)                                       # [pages, heads, positions, dim]
    there = (col[:, None] * P + torch.arange(P, device=dev) < kv_len[seq][:, None])[:, None, :, None]
    inf = torch.full((), math.inf, device=dev)
    out = st["bounds"].clone()
    out[ids] = torch.stack([torch.where(there, K, inf).amin(2), torch.where(there, K, -inf).amax(2)], 2).half()
    return {"bounds": out}


def _plain_select(st):
    case = st["case"]
    nkv, hd, P = case["kv_heads"], case["dim"], case["page"]
    seq, pos = _tokens(st)
    q = st["q"].float().unflatten(1, (nkv, -1))                                # [tokens, KV heads, group, dim]
    up = functools.reduce(torch.add, q.clamp(min=0).unbind(2))[:, None]
    down = functools.reduce(torch.add, q.clamp(max=0).unbind(2))[:, None]
    bounds = st["bounds"][st["table"].clamp(min=0).long()[seq]].float()        # [tokens, pages, KV heads, 2, dim]
    score = _eights(up * bounds[..., 1, :]) + _eights(down * bounds[..., 0, :])
    held = torch.where(pos >= 0, pos // P + 1, 0)
    pages, visible = _lists(score.transpose(1, 2), held, pos, st["table"][seq], case["budget"], P)
    return {"pages": pages, "visible": visible}


def _plain_attention(st):
    case = st["case"]
    nkv, hd, P = case["kv_heads"], case["dim"], case["page"]
    ids, heads = st["pages"].clamp(min=0).long(), torch.arange(nkv, device=st["q"].device)[None, :, None]
    K, V = (_held(st[w][ids, heads], P, hd).flatten(2, 3) for w in ("k_pages", "v_pages"))   # [tokens, heads, positions, dim]
    see = (torch.arange(K.shape[2], device=K.device)[None] < st["visible"][:, None])[:, None, :, None]
    K, V = (torch.where(see, x, torch.zeros((), device=K.device)) for x in (K, V))
    S = st["q"].float().unflatten(1, (nkv, -1)) @ K.transpose(2, 3) * (1.0 / math.sqrt(hd))
    S = torch.where(see.transpose(2, 3), S, torch.full((), -math.inf, device=K.device))
    top = S.amax(-1, keepdim=True)
    S = torch.exp(S - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = S.sum(-1, keepdim=True)
    return (S @ V / torch.where(total > 0, total, torch.ones_like(total))).flatten(1, 2).to(st["q"].dtype)


def _plain(st):
    op = st["case"]["op"]
    if op == "bounds":
        return _plain_bounds(st)
    if op == "select":
        return _plain_select(st)
    if op == "pages":
        return {"out": _plain_attention(st)}
    q = _turned(st["q"], st["q_gain"], st["pos"], st["axis"], st["rope"]).to(st["q"].dtype)
    k = _turned(st["k"], st["k_gain"], st["pos"], st["axis"], st["rope"])
    if op == "axes":
        return {"q": q, "k": k.to(st["k"].dtype)}
    return {"q": q, "k": _stored(k).half(), "v": _stored(st["v"]).half()}


# --------------------------------------------------------------------------- a pass
def run(st):
    if not own:
        return _plain(st)
    import paper_2606_09514_gb300 as pkg
    case = st["case"]
    op = case["op"]
    if op in ("axes", "append") and "axes" not in st:   # the layout that a program keeps with its model
        st["axes"] = pkg.buddy_rope_axes(case["dim"], [int(s) for s in case["sections"].split()], case["round"])
    if op == "axes":
        pkg.buddy_qk_norm_rope(st["q"], st["k"], st["pos"], st["rope"], st["q_out"], st["k_out"], st["q_gain"],
                               st["k_gain"], EPS, st["flags"], axes=st["axes"])
        return {"q": st["q_out"], "k": st["k_out"]}
    if "cache" not in st:   # the handle that a program keeps as long as its pages
        st["cache"] = pkg.KV4Cache(st["k_pages"], st["v_pages"], case["page"])
    cache = st["cache"]
    if op == "append":
        cache.buddy_kv4_append(st["q"], st["k"], st["v"], st["pos"], st["slot"], st["rope"], st["q_out"],
                               st["q_gain"], st["k_gain"], EPS, st["flags"], axes=st["axes"])
        cache.buddy_kv4_read(st["slot"], st["k_read"], st["v_read"], st["flags"])
        return {"q": st["q_out"], "k": st["k_read"], "v": st["v_read"]}
    if op == "bounds":
        cache.buddy_kv4_bounds(st["bounds"], st["kv_len"], st["table"], st["row_start"], st["max_new"], st["flags"])
        return {"bounds": st["bounds"]}
    if op == "select":
        cache.buddy_kv4_select(st["q"], st["bounds"], st["kv_len"], st["table"], st["pages"], st["visible"],
                               st["row_start"], st["max_new"], flags=st["flags"])
        return {"pages": st["pages"], "visible": st["visible"]}
    cache.buddy_kv4_attention_pages(st["q"], st["visible"], st["pages"], st["out"], flags=st["flags"])
    return {"out": st["out"]}


# --------------------------------------------------------------------------- in 64 bits
def _exact_turned(x, gain, pos, axis, rope):
    x = x.double()
    h = x.shape[-1] // 2
    if gain is not None:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * gain.double()
    j = torch.arange(h, device=x.device)
    turn = torch.complex(rope[0].double(), rope[1].double())
    z = torch.complex(x[..., :h], x[..., h:])
    for f in range(h):
        z[..., f] *= turn[pos[axis[f]].long(), j[f]][:, None]
    return torch.cat([z.real, z.imag], -1)


def _exact_stored(x):
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], GROUP):
        grp = x[..., c:c + GROUP]
        s = grp.abs().max(-1, keepdim=True).values / 7
        low = 2.0 ** (torch.floor(torch.log2(s.clamp(min=1e-30))) - 6)     # the last of seven bits
        s = (torch.round(s / low) * low).clamp(max=896.0)
        s = torch.round(s * 2.0 ** 24) / 2.0 ** 24                         # the smallest step of 16 bits
        out[..., c:c + GROUP] = torch.where(s > 0, torch.round(grp / s.clamp(min=1e-30)).clamp(-7, 7) * s, 0.0)
    return out


def _exact_values(blk, page, hd):
    """[n, positions, dim] of n blocks, byte by byte."""
    codes = blk[:, :page * hd // 2].reshape(-1, page, hd // 8, 4)
    scale = blk[:, page * hd // 2:].contiguous().view(torch.float16).reshape(-1, page, hd // GROUP)
    out = torch.empty(*codes.shape[:3], 8, dtype=torch.float64, device=blk.device)
    for j in range(8):
        ch = 2 * j if j < 4 else 2 * (j - 4) + 1
        out[..., ch] = ((codes[..., j // 2] >> (4 * (j % 2))) & 15).double() - 8
    return out.reshape(-1, page, hd) * scale.double().repeat_interleave(GROUP, -1)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    nq, nkv, hd, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    if op == "select":
        return None        # whole numbers: the plain form's have to be equal
    if op in ("axes", "append"):
        q = _exact_turned(st["q"], st["q_gain"], st["pos"], _axis_of(case), st["rope"])
        k = _exact_turned(st["k"], st["k_gain"], st["pos"], _axis_of(case), st["rope"])
        return {"q": q, "k": k} if op == "axes" else {"q": q, "k": _exact_stored(k), "v": _exact_stored(st["v"])}
    if op == "bounds":
        out = st["bounds"].double()
        for i, (n, m) in enumerate(zip(*_lengths(case))):
            full = n // P                       # pages that are written to their ends
            for a in range(max(0, n - m) // P, _ceil(n, P), 512):
                b = min(a + 512, _ceil(n, P))
                ids = st["table"][i, a:b].long()
                K = _exact_values(st["k_pages"][ids].flatten(0, 1), P, hd).unflatten(0, (-1, nkv))
                out[ids, :, 0], out[ids, :, 1] = K.min(2).values, K.max(2).values
                if b > full:
                    K = K[-1, :, :n % P]
                    out[ids[-1], :, 0], out[ids[-1], :, 1] = K.min(1).values, K.max(1).values
        return {"bounds": out}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    step = max(1, 100_000_000 // (nkv * case["budget"] * P * hd))
    heads = torch.arange(nkv, device=out.device)[None, :, None]
    for a in range(0, len(out), step):
        ids, n = st["pages"][a:a + step].clamp(min=0).long(), st["visible"][a:a + step]
        K, V = (_exact_values(st[w][ids, heads].flatten(0, 2), P, hd).reshape(len(ids), nkv, -1, hd)
                for w in ("k_pages", "v_pages"))
        hide = (torch.arange(K.shape[2], device=K.device)[None] >= n[:, None])[:, None, :]
        K, V = (x.masked_fill(hide[..., None], 0.0) for x in (K, V))
        s = torch.einsum("tgqd,tgpd->tgqp", st["q"][a:a + step].double().unflatten(1, (nkv, -1)), K) / math.sqrt(hd)
        p = torch.softmax(s.masked_fill(hide[..., None, :], -math.inf), -1)
        out[a:a + step] = torch.einsum("tgqp,tgpd->tgqd", p.nan_to_num(0.0), V).flatten(1, 2)
    return {"out": out}
