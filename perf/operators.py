"""Measured cases of the paged 4-bit cache's operators: what a serving program calls
between the projections of a block, through the package's public entry points.

A case is a dict of plain values:
  op       "plan" (buddy_page_plan), "norm" (buddy_qk_norm_rope), "append"
           (buddy_kv4_append, and buddy_kv4_read of what it stored) or
           "attention" (buddy_kv4_attention)
  batch    sequences (plan, attention)
  lo, hi   positions that a sequence holds before the call, spread over [lo, hi]
           (over their logarithm); every 16th sequence holds nothing
  new_lo, new_hi   new tokens per sequence (plan) or query tokens (attention)
  tokens   tokens of the call (norm, append)
  heads, kv_heads, dim   head layout
  page     positions per page
  dtype    "f32" or "bf16": type of q, k, v and the outputs
  gains    queries and keys are normalised for each head before the rotation
  spread   seed of the lengths: they belong to the case, the values to the seed
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
THETA = 1e6
GROUP = 32          # channels that share a scale
NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)   # channel of a word of eight -> nibble that holds it

# (query heads, KV heads, head dim): grouped heads of 128, as many KV heads as
# query heads, odd groups, heads of 64
HEADS = ((32, 8, 128), (28, 4, 128), (40, 40, 128), (6, 2, 128), (9, 3, 64), (4, 4, 64), (5, 1, 64))


# --------------------------------------------------------------------------- cases
def _plan(name, batch, lo, hi, new_lo, new_hi, page, spread):
    c = {"op": "plan", "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "page": page,
         "spread": spread}
    return {**c, "name": name} if name else c


def _rows(name, op, tokens, heads, dtype, gains, page=64):
    c = {"op": op, "tokens": tokens, "heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype,
         "gains": gains, "page": page}
    return {**c, "name": name} if name else c


def _attention(name, batch, lo, hi, new_lo, new_hi, heads, dtype, page, spread):
    c = {"op": "attention", "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi,
         "heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "dtype": dtype, "page": page, "spread": spread}
    return {**c, "name": name} if name else c


def listed():
    return [
        # the pages of a full server's next token
        _plan("plan-decode-250", 250, 512, 8192, 1, 1, 64, 1),
        # prompts that arrive together, in small pages
        _plan("plan-prompts-61", 61, 0, 0, 128, 1024, 16, 2),
        # one user's next token
        _rows("norm-1", "norm", 1, (32, 8, 128), "bf16", True),
        # a decode batch of a model in 32 bits
        _rows("norm-f32-250", "norm", 250, (28, 4, 128), "f32", True),
        # all tokens of 16 prompts
        _rows("norm-8297", "norm", 8297, (32, 8, 128), "bf16", True),
        # the new entries of a decode batch
        _rows("append-64", "append", 64, (32, 8, 128), "bf16", True, 64),
        # prompts of a model without the norms: rotation and 4 bits only
        _rows("append-4999", "append", 4999, (28, 4, 128), "bf16", False, 32),
        # one user's generation in a conversation of ordinary length
        _attention("decode-1-2048", 1, 2048, 2048, 1, 1, (32, 8, 128), "bf16", 64, 3),
        # one user's generation over a long document
        _attention("decode-1-120001", 1, 120001, 120001, 1, 1, (32, 8, 128), "bf16", 64, 4),
        # a full server, requests of all ages, idle slots among them
        _attention("decode-250", 250, 512, 8192, 1, 1, (28, 4, 128), "bf16", 64, 5),
        # several proposed tokens of each request checked at once; a KV head for each query head
        _attention("verify-31", 31, 100, 4096, 1, 5, (40, 40, 128), "bf16", 16, 6),
        # pieces of prompts over what their requests hold already, next to single tokens
        _attention("prompts-9", 9, 300, 6000, 1, 1500, (32, 8, 128), "bf16", 128, 7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(("plan", "norm", "append", "attention", "attention"))
    heads, page, dtype = rng.choice(HEADS), rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "bf16", "f32"))
    spread = rng.randrange(1 << 20)
    if op == "plan":
        batch = _log(rng, 1, 1000)
        new = _log(rng, 1, min(1024, 65536 // batch))
        hi = rng.choice((0, _log(rng, 1, 8192)))
        return _plan(None, batch, min(hi, 512), hi, max(1, new // 4), new, page, spread)
    if op in ("norm", "append"):
        # a layout of 40 + 80 heads moves four times what 28 + 8 do
        t = _log(rng, 1, 4000 if op == "append" else 8000)
        return _rows(None, op, max(1, t * 8 // max(8, heads[1])), heads, dtype, rng.random() < 0.7, page)
    # attention: (sequence, KV head, position) triples within what decode-250 has,
    # (token, position) pairs within what prompts-9 has
    dtype = "bf16"
    kind = rng.choice(("decode", "decode", "verify", "prompts"))
    triples = 2_000_000 * 128 // heads[2] // heads[1]
    if kind == "prompts":
        batch, new = _log(rng, 1, 8), _log(rng, 20, 1200)
        hi = _log(rng, 1, max(2, min(40000, 8_000_000 * 32 // (batch * new * heads[0]))))
        return _attention(None, batch, max(1, hi // 8), hi, max(1, new // 16), new, heads, dtype, page, spread)
    batch = _log(rng, 1, 250)
    hi = _log(rng, 1, max(2, min(100000, triples // batch)))
    new = 1 if kind == "decode" else rng.randint(2, 8)
    return _attention(None, batch, max(1, hi // 16), hi, 1, new, heads, dtype, page, spread)


def _lengths(case):
    """Positions held before the call and new tokens of each sequence."""
    rng = random.Random("lengths %d" % case["spread"])
    held, new = [], []
    for i in range(case["batch"]):
        n = 0 if case["hi"] == 0 else _log(rng, max(1, case["lo"]), case["hi"])
        m = rng.randint(case["new_lo"], case["new_hi"])
        if i % 16 == 15:      # an idle slot: nothing held; a plan gives it no token either
            n, m = 0, 0 if case["op"] == "plan" else m
        elif i % 4 == 3:      # a request that decodes next to the others' longer pieces
            m = case["new_lo"]
        held.append(n)
        new.append(m)
    if case["op"] == "attention" and case["batch"] > 1:   # the longest piece there is
        new[0] = case["new_hi"]
    return held, new


def _visible(case):
    """Cached positions of each sequence, new ones among them; idle slots: 0."""
    held, new = _lengths(case)
    return [h + n if i % 16 != 15 else 0 for i, (h, n) in enumerate(zip(held, new))], new


def _pages(n, page):
    return -(-n // page)


def work(case):
    op = case["op"]
    if op == "plan":
        held, new = _lengths(case)
        pages = sum(_pages(h + n, case["page"]) - _pages(h, case["page"]) for h, n in zip(held, new))
        return {"bytes": 16 * case["batch"] + 8 * pages + 12 * sum(new), "flops": 0}
    nq, nkv, hd = case["heads"], case["kv_heads"], case["dim"]
    e = 4 if case["dtype"] == "f32" else 2
    entry = hd // 2 + hd // 16
    if op in ("norm", "append"):
        t = case["tokens"]
        rotated = nq + nkv
        b = t * (rotated * hd * e + hd * 4 + 4)                       # q, k, cos and sin, positions
        if op == "norm":
            return {"bytes": b + t * rotated * hd * e, "flops": t * rotated * hd * 10}
        b += t * (nkv * hd * e + nq * hd * e + 8 + 2 * nkv * entry)    # v, q's output, slots, the entries stored
        b += t * (8 + 2 * nkv * entry + 2 * nkv * hd * 2)              # the entries read back, and their values
        return {"bytes": b, "flops": t * (rotated * hd * 10 + 2 * nkv * hd * 4)}
    have, new = _visible(case)
    pairs = sum(sum(max(0, h - n + j + 1) for j in range(n)) for h, n in zip(have, new))
    return {"bytes": sum(have) * nkv * 2 * entry + 2 * sum(new) * nq * hd * e + 12 * case["batch"],
            "flops": 4 * nq * hd * pairs}


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


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    op = case["op"]
    st = {"case": case, "flags": torch.zeros(1, dtype=torch.int32, device=dev)}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    if op == "plan":
        held, new = _lengths(case)
        P, B = case["page"], case["batch"]
        row = max(_pages(h + n, P) for h, n in zip(held, new)) + 3
        have = [_pages(h, P) for h in held]
        pool = sum(_pages(h + n, P) for h, n in zip(held, new)) + 100
        ids = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
        table = torch.full((B, row), -1, dtype=torch.int32, device=dev)
        at = torch.arange(row, device=dev)[None] < i32(have)[:, None]
        table[at] = ids[:sum(have)]
        free = ids[sum(have):].contiguous()
        st.update(length=i32(held), n_new=i32(new), table=table, free=torch.cat([i32([7, 7, 7]), free]),
                  head=i32([3]), head_out=i32([0]), kv_len=torch.empty(B, dtype=torch.int32, device=dev),
                  row_start=torch.empty(B + 1, dtype=torch.int32, device=dev),
                  slot=torch.empty(sum(new), dtype=torch.int64, device=dev),
                  pos=torch.empty(sum(new), dtype=torch.int32, device=dev))
        return st
    nq, nkv, hd, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    if op in ("norm", "append"):
        t = case["tokens"]
        # one projection's output: queries, keys and values of a token side by side;
        # some channels of the keys are larger than the others
        qkv = torch.randn(t, (nq + 2 * nkv) * hd, generator=g, device=dev)
        qkv[:, nq * hd:(nq + nkv) * hd] *= torch.exp(0.4 * torch.randn(nkv * hd, generator=g, device=dev))
        qkv = qkv.to(dt)
        st.update(q=qkv[:, :nq * hd].unflatten(1, (nq, hd)), k=qkv[:, nq * hd:(nq + nkv) * hd].unflatten(1, (nkv, hd)),
                  v=qkv[:, (nq + nkv) * hd:].unflatten(1, (nkv, hd)), rope=_rope(8320, hd, dev),
                  pos=torch.randint(0, 8320, (t,), generator=g, device=dev, dtype=torch.int32),
                  q_gain=None, k_gain=None, q_out=torch.empty(t, nq, hd, dtype=dt, device=dev))
        if case["gains"]:
            st["q_gain"] = torch.rand(hd, generator=g, device=dev) + 0.5
            st["k_gain"] = torch.rand(hd, generator=g, device=dev) + 0.5
        if op == "norm":
            st["k_out"] = torch.empty(t, nkv, hd, dtype=dt, device=dev)
            return st
        # up to 256 tokens: one per request, each in a page of its own; above: prompts,
        # position by position through pages that lie anywhere
        n_pages = (t if t <= 256 else _pages(t, page)) + 20
        st["k_pages"], st["v_pages"] = (_random_pages(n_pages, nkv, page, hd, g, dev) for _ in range(2))
        ids = torch.randperm(n_pages, generator=g, device=dev)
        if t <= 256:
            st["slot"] = ids[:t] * page + torch.randint(0, page, (t,), generator=g, device=dev)
        else:
            st["slot"] = (ids[:, None] * page + torch.arange(page, device=dev)).reshape(-1)[:t].contiguous()
        st["k_read"], st["v_read"] = (torch.empty(t, nkv, hd, dtype=torch.float16, device=dev) for _ in range(2))
        return st
    have, new = _visible(case)
    row = max(1, max(_pages(n, page) for n in have)) + 1
    need = sum(_pages(n, page) for n in have)
    n_pages = need + 10
    st["k_pages"], st["v_pages"] = (_random_pages(n_pages, nkv, page, hd, g, dev) for _ in range(2))
    table = torch.full((case["batch"], row), -1, dtype=torch.int32, device=dev)
    used = torch.arange(row, device=dev)[None] < i32([_pages(n, page) for n in have])[:, None]
    table[used] = torch.randperm(n_pages, generator=g, device=dev)[:need].to(torch.int32)
    # what no request has written yet is what the memory held: NaN scales here, behind the
    # last position of each sequence
    for i, n in enumerate(have):
        if n % page:
            p = int(table[i, n // page])
            for pages in (st["k_pages"], st["v_pages"]):
                pages[p, :, page * hd // 2:].unflatten(1, (page, hd // 16))[:, n % page:] = 0xFF
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    st.update(q=(2 * torch.randn(starts[-1], nq, hd, generator=g, device=dev)).to(dt), table=table,
              kv_len=i32(have), row_start=i32(starts) if case["new_hi"] > 1 else None, max_new=max(new),
              out=torch.empty(starts[-1], nq, hd, dtype=dt, device=dev))
    return st


# --------------------------------------------------------------------------- plain form
def _halve(y):
    """Sum over the last axis: the upper half onto the lower, until one is left."""
    n = y.shape[-1]
    return y[..., 0] if n == 1 else _halve(y[..., :n // 2] + y[..., n // 2:])


def _turned(x, gain, pos, rope):
    """Norm of each head (where there are gains) and rotation, in 32 bits."""
    x = x.float()
    if gain is not None:
        # the order of the sum is a part of the operator's definition: eight
        # neighbours, then the eights
        total = _halve(_halve((x * x).unflatten(-1, (-1, 8))))
        x = x * (1.0 / torch.sqrt(total * (1.0 / x.shape[-1]) + EPS))[..., None] * gain
    c, s = rope[0][pos.long()][:, None], rope[1][pos.long()][:, None]
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


def _held(pages, table, page, hd):
    """The values of each sequence's pages: [batch, positions, KV heads, dim] in 32 bits."""
    blk = pages[table.clamp(min=0).long()]                                     # [B, pages, heads, bytes]
    B, n, h = blk.shape[:3]
    codes, scales = blk[..., :page * hd // 2], blk[..., page * hd // 2:].contiguous().view(torch.float16)
    nib = torch.stack([codes & 15, codes >> 4], -1).reshape(B, n, h, page, hd // 8, 8)
    val = nib[..., list(NIBBLE)].reshape(B, n, h, page, hd // GROUP, GROUP).float() - 8.0
    val = val * scales.reshape(B, n, h, page, hd // GROUP, 1).float()
    return val.reshape(B, n, h, page, hd).transpose(2, 3).reshape(B, n * page, h, hd)


def _plain_plan(st):
    P, table = st["case"]["page"], st["table"]
    length, new = st["length"].long(), st["n_new"].long()
    dev, T = length.device, st["slot"].shape[0]
    have, after = (length + P - 1) // P, (length + new + P - 1) // P
    ends = torch.cumsum(after - have, 0)
    first = st["head"].long() + ends - (after - have)           # each sequence's first new page in the list
    col = torch.arange(table.shape[1], device=dev)[None]
    at = first[:, None] + col - have[:, None]
    fresh = (col >= have[:, None]) & (col < after[:, None])
    table = torch.where(fresh, st["free"][at.clamp(0, st["free"].shape[0] - 1)], table)
    starts = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    t = torch.arange(T, device=dev)
    seq = (t[:, None] >= starts[None, 1:]).sum(1)
    pos = length[seq] + t - starts[seq]
    slot = table[seq, pos // P].long() * P + pos % P
    return {"table": table, "kv_len": (length + new).int(), "row_start": starts.int(), "slot": slot,
            "pos": pos.int(), "head": st["head"] + ends[-1:].int()}


def _plain_attention(st):
    case = st["case"]
    nq, nkv, hd, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    q, kv_len, B, dev = st["q"], st["kv_len"].long(), case["batch"], st["q"].device
    start = torch.arange(B + 1, device=dev) if st["row_start"] is None else st["row_start"].long()
    new, most, T = start[1:] - start[:-1], st["max_new"], q.shape[0]
    K, V = _held(st["k_pages"], st["table"], page, hd), _held(st["v_pages"], st["table"], page, hd)
    L = K.shape[1]
    there = torch.arange(L, device=dev)[None] < kv_len[:, None]
    K, V = (torch.where(there[:, :, None, None], x, torch.zeros((), device=dev)) for x in (K, V))
    j = torch.arange(most, device=dev)
    Q = q[(start[:-1, None] + j).clamp(max=T - 1)].float()                     # [B, most, nq, hd]
    Q = Q.reshape(B, most, nkv, nq // nkv, hd).permute(0, 2, 1, 3, 4).reshape(B, nkv, -1, hd)
    S = Q @ K.permute(0, 2, 3, 1) * (1.0 / math.sqrt(hd))                      # [B, nkv, most * group, L]
    last = (kv_len - new)[:, None] + j                                         # each query's own position
    see = torch.arange(L, device=dev)[None, None] <= last[..., None]           # [B, most, L]
    see = (see & there[:, None]).repeat_interleave(nq // nkv, 1)[:, None]
    S = torch.where(see, S, torch.full((), -math.inf, device=dev))
    top = S.amax(-1, keepdim=True)
    S = torch.exp(S - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = S.sum(-1, keepdim=True)
    O = S @ V.permute(0, 2, 1, 3) / torch.where(total > 0, total, torch.ones_like(total))
    O = O.reshape(B, nkv, most, nq // nkv, hd).permute(0, 2, 1, 3, 4).reshape(B, most, nq, hd)
    t = torch.arange(T, device=dev)
    seq = (t[:, None] >= start[None, 1:]).sum(1)
    return O[seq, t - start[seq]].to(q.dtype)


def _plain(st):
    op = st["case"]["op"]
    if op == "plan":
        return _plain_plan(st)
    if op == "attention":
        return {"out": _plain_attention(st)}
    q = _turned(st["q"], st["q_gain"], st["pos"], st["rope"]).to(st["q"].dtype)
    k = _turned(st["k"], st["k_gain"], st["pos"], st["rope"])
    if op == "norm":
        return {"q": q, "k": k.to(st["k"].dtype)}
    return {"q": q, "k": _stored(k).half(), "v": _stored(st["v"]).half()}


# --------------------------------------------------------------------------- a pass
def run(st):
    if not own:
        return _plain(st)
    import paper_2606_09514_gb300 as pkg
    case = st["case"]
    op = case["op"]
    if op == "plan":
        pkg.buddy_page_plan(st["length"], st["n_new"], case["page"], st["table"], st["free"], st["head"],
                            st["kv_len"], st["row_start"], st["slot"], st["pos"], st["head_out"], st["flags"])
        return {"table": st["table"], "kv_len": st["kv_len"], "row_start": st["row_start"], "slot": st["slot"],
                "pos": st["pos"], "head": st["head_out"]}
    if op == "norm":
        pkg.buddy_qk_norm_rope(st["q"], st["k"], st["pos"], st["rope"], st["q_out"], st["k_out"], st["q_gain"],
                               st["k_gain"], EPS, st["flags"])
        return {"q": st["q_out"], "k": st["k_out"]}
    if "cache" not in st:   # the handle that a program keeps as long as its pages
        st["cache"] = pkg.KV4Cache(st["k_pages"], st["v_pages"], case["page"])
    cache = st["cache"]
    if op == "append":
        cache.buddy_kv4_append(st["q"], st["k"], st["v"], st["pos"], st["slot"], st["rope"], st["q_out"],
                               st["q_gain"], st["k_gain"], EPS, st["flags"])
        cache.buddy_kv4_read(st["slot"], st["k_read"], st["v_read"], st["flags"])
        return {"q": st["q_out"], "k": st["k_read"], "v": st["v_read"]}
    cache.buddy_kv4_attention(st["q"], st["kv_len"], st["table"], st["out"], st["row_start"], st["max_new"],
                              flags=st["flags"])
    return {"out": st["out"]}


# --------------------------------------------------------------------------- in 64 bits
def _exact_turned(x, gain, pos, rope):
    x = x.double()
    h = x.shape[-1] // 2
    if gain is not None:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS) * gain.double()
    z = torch.complex(x[..., :h], x[..., h:]) * torch.complex(rope[0].double(), rope[1].double())[pos.long()][:, None]
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


def _exact_values(pages, ids, page, hd):
    """[heads, positions, dim] of one sequence's pages, byte by byte."""
    blk = pages[ids.long()].permute(1, 0, 2)                                   # [heads, pages, bytes]
    codes = blk[..., :page * hd // 2].reshape(*blk.shape[:2], page, hd // 8, 4)
    scale = blk[..., page * hd // 2:].contiguous().view(torch.float16).reshape(*blk.shape[:2], page, hd // GROUP)
    out = torch.empty(*codes.shape[:4], 8, dtype=torch.float64, device=pages.device)
    for j in range(8):
        ch = 2 * j if j < 4 else 2 * (j - 4) + 1
        out[..., ch] = ((codes[..., j // 2] >> (4 * (j % 2))) & 15).double() - 8
    out = out.reshape(*blk.shape[:2], page, hd) * scale.double().repeat_interleave(GROUP, -1)
    return out.flatten(1, 2)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "plan":
        return None        # whole numbers: the plain form's have to be equal
    if op in ("norm", "append"):
        q = _exact_turned(st["q"], st["q_gain"], st["pos"], st["rope"])
        k = _exact_turned(st["k"], st["k_gain"], st["pos"], st["rope"])
        return {"q": q, "k": k} if op == "norm" else {"q": q, "k": _exact_stored(k), "v": _exact_stored(st["v"])}
    have, new = _visible(case)
    nq, nkv, hd, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    at = 0
    for i, (n, m) in enumerate(zip(have, new)):
        if n:
            ids = st["table"][i, :_pages(n, page)]
            K, V = (_exact_values(st[w], ids, page, hd)[:, :n] for w in ("k_pages", "v_pages"))
            p = torch.arange(n, device=K.device)
            for a in range(0, m, 512):
                b = min(m, a + 512)
                q = st["q"][at + a:at + b].double().reshape(b - a, nkv, nq // nkv, hd)
                s = torch.einsum("tghd,gpd->gthp", q, K) / math.sqrt(hd)
                hide = p[None] > (n - m + torch.arange(a, b, device=K.device))[:, None]
                s.masked_fill_(hide[None, :, None], -math.inf)
                out[at + a:at + b] = torch.einsum("gthp,gpd->tghd", torch.softmax(s, -1), V).reshape(b - a, nq, hd)
        at += m
    return {"out": out}
