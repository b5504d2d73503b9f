"""Serving over a paged 4-bit cache: pieces of prompts next to single tokens.

A stack of attention layers (norm of the residual, one projection for queries, keys and
values, norm of each head and rotation, attention, output projection) whose sequences share
a pool of pages.  Every call runs

    buddy_page_plan       pages, slots and positions of the call's tokens, once for all layers
    buddy_kv4_append      per layer: head norms, rotation, keys and values to 4 bits
    buddy_kv4_attention   per layer: the call's queries over everything stored

and the lengths advance on the GPU; the host only knows how many tokens a call has.  A sequence
takes its prompt in pieces while those whose prompts were shorter go on token by token; when all
are through, the step is captured in a CUDA graph.  Weights are random.  At the end the last
layer's outputs of the last step are compared with attention in 64 bits over the entries read
back, and what the stack has added to the last tokens with the same stack without a cache, over
everything that the sequences were fed: with keys and values rounded to 4 bits as the cache
rounds them (the rest is bf16's roundings), and with exact ones (what the 4 bits cost).

    python examples/serve_kv4.py [--layers 4] [--batch 8] [--prompt 600] [--piece 128] [--steps 32]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_09514_gb300 as buddy  # noqa: E402

D, NQ, NKV, HD, PAGE, EPS, THETA = 1024, 16, 4, 64, 64, 1e-6, 1e6


class Server:
    def __init__(self, layers: int, batch: int, max_len: int, device="cuda"):
        self.batch, self.device = batch, device
        self.max_pages = -(-max_len // PAGE)
        i32 = dict(dtype=torch.int32, device=device)
        n_pages = batch * self.max_pages
        self.length, self.kv_len = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.row_start = torch.zeros(batch + 1, **i32)
        self.table = torch.full((batch, self.max_pages), -1, **i32)
        self.free = torch.randperm(n_pages, device=device).to(torch.int32)
        self.head, self.head_out = torch.zeros(1, **i32), torch.zeros(1, **i32)
        self.flags = torch.zeros(1, **i32)
        self.rope = buddy.buddy_rope_table(max_len, HD, THETA, device)
        width = (NQ + 2 * NKV) * HD
        bf16 = dict(dtype=torch.bfloat16, device=device)
        self.w_qkv = [torch.randn(D, width, **bf16) / math.sqrt(D) for _ in range(layers)]
        self.w_o = [torch.randn(NQ * HD, D, **bf16) / math.sqrt(NQ * HD) for _ in range(layers)]
        self.gains = [[torch.rand(HD, device=device) + 0.5 for _ in range(2)] for _ in range(layers)]
        self.caches = [buddy.KV4Cache.empty(n_pages, PAGE, NKV, HD, device) for _ in range(layers)]
        # the layers run one after the other: one workspace serves them all
        ws = torch.zeros(self.caches[0].workspace_bytes(NQ, max_len), dtype=torch.uint8, device=device)
        for c in self.caches:
            c.workspace = ws

    def forward(self, x: torch.Tensor, n_new: torch.Tensor, max_new: int) -> torch.Tensor:
        """x [tokens, D]: the new tokens of every sequence, sequence by sequence."""
        T = x.shape[0]
        slot = torch.empty(T, dtype=torch.int64, device=self.device)
        pos = torch.empty(T, dtype=torch.int32, device=self.device)
        buddy.buddy_page_plan(self.length, n_new, PAGE, self.table, self.free, self.head, self.kv_len, self.row_start,
                              slot, pos, self.head_out, self.flags)
        for w_qkv, w_o, (q_gain, k_gain), cache in zip(self.w_qkv, self.w_o, self.gains, self.caches):
            h = x.float()
            h = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)).to(x.dtype)
            q, k, v = (h @ w_qkv).unflatten(1, (NQ + 2 * NKV, HD)).split((NQ, NKV, NKV), 1)
            q_out, out = torch.empty(2, T, NQ, HD, dtype=x.dtype, device=self.device)
            cache.buddy_kv4_append(q, k, v, pos, slot, self.rope, q_out, q_gain, k_gain, EPS, self.flags)
            cache.buddy_kv4_attention(q_out, self.kv_len, self.table, out, self.row_start, max_new, flags=self.flags)
            x = x + out.flatten(1) @ w_o
            self.last = (q_out, out)
        self.length.copy_(self.kv_len)
        self.head.copy_(self.head_out)
        return x

    def check(self) -> float:
        """Largest deviation of the last layer's last single-token outputs from 64 bits."""
        q, out = self.last
        worst = 0.0
        for i in range(self.batch):
            n = int(self.kv_len[i])
            p = torch.arange(n, device=self.device)
            slot = self.table[i].long()[p // PAGE] * PAGE + p % PAGE
            k, v = torch.empty(2, n, NKV, HD, device=self.device)
            self.caches[-1].buddy_kv4_read(slot, k, v)
            k, v = (x.double().repeat_interleave(NQ // NKV, 1) for x in (k, v))
            s = torch.softmax(torch.einsum("hd,phd->hp", q[i].double(), k) / math.sqrt(HD), -1)
            want = torch.einsum("hp,phd->hd", s, v)
            worst = max(worst, float((out[i].double() - want).abs().max() / want.abs().max()))
        return worst


def four_bits(x: torch.Tensor) -> torch.Tensor:
    """What the cache holds of x [..., HD] fp32 (finite values)."""
    g = x.unflatten(-1, (-1, 32))
    s = g.abs().amax(-1, keepdim=True) / 7
    m, e = torch.frexp(s)
    s = torch.ldexp((m * 128).round(), e - 7).clamp(max=896).half().float()    # 7 significant bits
    return torch.where(s > 0, (g / s).round().clamp(-7, 7) * s, 0.0).flatten(-2)


def without_cache(s: Server, x: torch.Tensor, rounded) -> torch.Tensor:
    """The stack over one whole sequence x [n, D], keys and values through `rounded`."""
    n = x.shape[0]
    co, si = (t[:n, None] for t in s.rope)
    seen = torch.ones(n, n, dtype=torch.bool, device=x.device).tril()

    def turned(v, gain):
        v = v.float()
        v = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * gain
        a, b = v.chunk(2, -1)
        return torch.cat([a * co - b * si, b * co + a * si], -1)

    for w_qkv, w_o, (q_gain, k_gain) in zip(s.w_qkv, s.w_o, s.gains):
        h = x.float()
        h = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)).to(x.dtype)
        q, k, v = (h @ w_qkv).unflatten(1, (NQ + 2 * NKV, HD)).split((NQ, NKV, NKV), 1)
        q = turned(q, q_gain).to(x.dtype).float()
        k, v = (rounded(t).repeat_interleave(NQ // NKV, 1) for t in (turned(k, k_gain), v.float()))
        p = (torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(HD)).masked_fill(~seen, -math.inf).softmax(-1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).to(x.dtype).flatten(1) @ w_o
    return x


def serve(argv=None) -> dict:
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=600, help="longest prompt")
    ap.add_argument("--piece", type=int, default=128, help="tokens of a prompt per call")
    ap.add_argument("--steps", type=int, default=32, help="single tokens after the longest prompt")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    # (a sequence gets a token in every call from its prompt's end on)
    s = Server(a.layers, a.batch, a.prompt + -(-a.prompt // a.piece) + a.steps + 8)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    left = [max(1, a.prompt * (i + 1) // a.batch) for i in range(a.batch)]
    fed = [[] for _ in left]
    mixed = 0
    while any(left):
        new = [min(a.piece, n) if n else 1 for n in left]
        mixed += 0 in left
        x = torch.randn(sum(new), D, **bf16)
        for f, part in zip(fed, x.split(new)):
            f.append(part)
        s.forward(x, torch.tensor(new, dtype=torch.int32, device="cuda"), max(new))
        left = [max(0, n - a.piece) for n in left]
    one = torch.ones(a.batch, dtype=torch.int32, device="cuda")
    x = torch.randn(a.batch, D, **bf16)
    s.forward(x, one, 1)                       # outside the graph first
    steps = [x.clone()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = s.forward(x, one, 1)
    for _ in range(a.steps):
        x.copy_(torch.randn_like(x))           # stands in for the rest of a model
        steps.append(x.clone())
        graph.replay()
    torch.cuda.synchronize()
    if s.flags.item():
        raise RuntimeError(f"device flags {s.flags.item()}")
    off = {}
    for what, rounded in (("model", four_bits), ("exact", lambda t: t)):
        got, want = [], []
        for i in range(a.batch):
            z = torch.cat(fed[i] + [t[i:i + 1] for t in steps])
            want.append((without_cache(s, z, rounded)[-1] - z[-1]).double())
            got.append((y[i] - x[i]).double())
        got, want = torch.stack(got), torch.stack(want)
        off[what] = float((got - want).norm() / want.norm())
    return {"tokens": int(s.length.sum()), "pages": int(s.head.item()), "mixed": mixed, "read": s.check(), **off}


def main(argv=None) -> float:
    r = serve(argv)
    print(f"{r['tokens']} positions in {r['pages']} pages of {PAGE}; {2 * NKV * (HD // 2 + HD // 16)} bytes per position and layer "
          f"(bf16: {2 * NKV * HD * 2}); {r['mixed']} calls with pieces of prompts next to single tokens; outputs within "
          f"{r['read']:.1e} of 64 bits over the entries, the stack's within {r['model']:.1e} of one without a cache "
          f"(4-bit entries; exact ones {r['exact']:.1e})")
    return r["read"]


if __name__ == "__main__":
    main()
