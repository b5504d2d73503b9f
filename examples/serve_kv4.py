"""Serving over a paged 4-bit cache: prompts of different lengths, then single tokens.

A stack of attention layers (norm of the residual, one projection for queries, keys and
values, norm of each head and rotation, attention, output projection) whose sequences share
a pool of pages.  Every call runs

    buddy_page_plan       pages, slots and positions of the call's tokens, once for all layers
    buddy_kv4_append      per layer: head norms, rotation, keys and values to 4 bits
    buddy_kv4_attention   per layer: the call's queries over everything stored

and the lengths advance on the GPU; the host only knows how many tokens a call has.
The decode step is captured in a CUDA graph.  Weights are random.  At the end the last layer's
outputs of the last step are compared with attention in 64 bits over the entries read back.

    python examples/serve_kv4.py [--layers 4] [--batch 8] [--prompt 600] [--steps 32]
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


def main(argv=None) -> float:
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=600, help="longest prompt")
    ap.add_argument("--steps", type=int, default=32, help="decode steps")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    s = Server(a.layers, a.batch, a.prompt + a.steps + 8)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    lengths = [max(1, a.prompt * (i + 1) // a.batch) for i in range(a.batch)]
    s.forward(torch.randn(sum(lengths), D, **bf16), torch.tensor(lengths, dtype=torch.int32, device="cuda"), max(lengths))
    one = torch.ones(a.batch, dtype=torch.int32, device="cuda")
    x = torch.randn(a.batch, D, **bf16)
    s.forward(x, one, 1)                       # outside the graph first
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = s.forward(x, one, 1)
    for _ in range(a.steps):
        x.copy_(y + torch.randn_like(y))       # stands in for the rest of a model
        graph.replay()
    torch.cuda.synchronize()
    if s.flags.item():
        raise RuntimeError(f"device flags {s.flags.item()}")
    tokens, pages = int(s.length.sum()), int(s.head.item())
    worst = s.check()
    print(f"{tokens} positions in {pages} pages of {PAGE}; {2 * NKV * (HD // 2 + HD // 16)} bytes per position and layer "
          f"(bf16: {2 * NKV * HD * 2}); outputs within {worst:.1e} of 64 bits")
    return worst


if __name__ == "__main__":
    main()
