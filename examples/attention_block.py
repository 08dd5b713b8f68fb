#!/usr/bin/env python3
"""The attention block of a decoder layer on this library alone: any4 QKV and O projections, a paged key-value cache of 16, 8 or 4 bits,
prompts (whole, or in parts behind what the cache already holds) and single tokens.

    python examples/attention_block.py [--bits 8] [--requests 4] [--prompt 700] [--tokens 16] [--window 256 [--sinks 4]] [--separate]

Sizes are Llama-3-8B's (hidden 4096, 32 query heads on 8 KV heads of 128), weights and inputs synthetic.  It feeds each request a prompt in
two parts and then token after token, and says how far the outputs are from the same block computed in one piece in 32 bits.
A layer is one call that turns q and k by their positions and writes k and v into the cache, and one of attention over the cache's pages.
With --separate PyTorch does the rotary embedding, and a prompt's later part reads its context out of the cache first.  PyTorch does the
bookkeeping of pages.
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
import paper_2507_04610_amd as any4  # noqa: E402
from paper_2507_04610_amd import inputs  # noqa: E402


def rotate(x, positions, base=500000.0):
    """rotary embedding of x [tokens, heads, dim] at positions [tokens]"""
    half = x.shape[-1] // 2
    angle = positions[:, None].float() * base ** (-torch.arange(half, device=x.device).float() / half)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat((a * c - b * s, b * c + a * s), -1).to(x.dtype)


class Linear:
    """a 4-bit linear with a table for each row, synthetic"""

    def __init__(self, n, k, seed, device="cuda"):
        t = inputs.make_case_device(1, n, k, 4, seed, device=device)
        self.codes = any4.any4_pack(t["codes_u8"], 4)
        self.lut, self.scale, self.offset = t["lut"], t["scale"], t["offset"]

    def __call__(self, x):
        return any4.any4_gemm(x, self.codes, self.lut, self.scale, self.offset, 4)


class AttentionBlock:
    """hidden -> heads of q, k, v -> attention over everything a request has had so far -> hidden"""

    def __init__(self, hidden=4096, heads=32, kv_heads=8, head_dim=128, pages=256, page_size=64, bits=8, max_pages=64, requests=4, device="cuda"):
        self.heads, self.kv_heads, self.dim, self.bits, self.page = heads, kv_heads, head_dim, bits, page_size
        self.qkv = Linear((heads + 2 * kv_heads) * head_dim, hidden, 1, device)
        self.o = Linear(hidden, heads * head_dim, 2, device)
        self.cache_k, self.cache_v, self.scales = any4.any4_kv_cache(pages, kv_heads, head_dim, page_size, bits, device=device)
        self.free = list(range(pages))[::-1]
        self.table = torch.zeros((requests, max_pages), dtype=torch.int32)             # on the host; sent along with each call
        self.lengths = [0] * requests
        self.device = device

    def _slots(self, request, start, end):
        t = torch.arange(start, end)
        return self.table[request, t // self.page].long() * self.page + t % self.page

    def _grow(self, request, tokens):
        """room for more tokens of a request; their slots"""
        start, end = self.lengths[request], self.lengths[request] + tokens
        for p in range(-(-start // self.page), -(-end // self.page)):
            self.table[request, p] = self.free.pop()
        self.lengths[request] = end
        return self._slots(request, start, end)

    def _project(self, x, positions, slots):
        row = self.qkv(x)
        n, h, g, d = x.shape[0], self.heads, self.kv_heads, self.dim
        q, k = rotate(row[:, :h * d].view(n, h, d), positions), rotate(row[:, h * d:(h + g) * d].view(n, g, d), positions)
        v = row[:, (h + g) * d:].view(n, g, d)                                          # (as it lies in the projection's rows)
        any4.any4_kv_write(k, v, slots.to(self.device), self.cache_k, self.cache_v, self.scales, bits=self.bits)
        return q, k, v

    def prompt(self, x, tokens):
        """x: rows of the requests' new tokens, packed, tokens[r] of request r, which may have had others before"""
        before = list(self.lengths)
        slots = torch.cat([self._grow(r, n) for r, n in enumerate(tokens)])
        positions = torch.cat([torch.arange(b, b + n) for b, n in zip(before, tokens)]).to(self.device)
        q, k, v = self._project(x, positions, slots)
        starts = lambda lengths: torch.tensor([0] + list(lengths), dtype=torch.int32).cumsum(0).to(torch.int32).to(self.device)      # noqa: E731
        if any(before):
            everything = torch.cat([self._slots(r, 0, n) for r, n in enumerate(self.lengths)]).to(self.device)
            k, v = any4.any4_kv_read(self.cache_k, self.cache_v, everything, self.scales, bits=self.bits, dtype=x.dtype)
        out = any4.any4_attn_prompt(q, k, v, starts(tokens), starts(self.lengths))
        return self.o(out.view(x.shape[0], -1))

    def token(self, x):
        """x: one row for each request"""
        positions = torch.tensor(self.lengths, device=self.device)
        slots = torch.cat([self._grow(r, 1) for r in range(x.shape[0])])
        q, _, _ = self._project(x, positions, slots)
        out = any4.any4_attn_decode(q, self.cache_k, self.cache_v, self.table.to(self.device),
                                    torch.tensor(self.lengths, dtype=torch.int32, device=self.device), self.scales, bits=self.bits)
        return self.o(out.view(x.shape[0], -1))

    def plain(self, x, weights):
        """one request's rows in one piece, causal, in 32 bits and without a cache; weights: those of qkv and o, dequantised"""
        n, h, g, d = x.shape[0], self.heads, self.kv_heads, self.dim
        row = x.float() @ weights[0].T
        at = torch.arange(n, device=x.device)
        q, k = rotate(row[:, :h * d].view(n, h, d), at), rotate(row[:, h * d:(h + g) * d].view(n, g, d), at)
        v = row[:, (h + g) * d:].view(n, g, d)
        k, v = k.repeat_interleave(h // g, 1), v.repeat_interleave(h // g, 1)
        out = torch.empty_like(q)
        for j in range(h):
            s = (q[:, j] @ k[:, j].T.contiguous()) * d ** -0.5
            out[:, j] = torch.softmax(s.masked_fill(~self._sees(at), float("-inf")), -1) @ v[:, j]
        return out.reshape(n, -1) @ weights[1].T

    def _sees(self, at):
        return at[:, None] >= at


class FusedBlock(AttentionBlock):
    """the same in two calls between the projections, prompts and single tokens alike; with a window, a token sees only the last `window` and
    the first `sinks`"""

    def __init__(self, *args, window=None, sinks=0, base=500000.0, **kw):
        super().__init__(*args, **kw)
        self.part = {} if window is None else dict(window=window, sinks=sinks)
        self.freqs = base ** (-torch.arange(self.dim // 2, dtype=torch.float64, device=self.device) / (self.dim // 2))

    def _project(self, x, positions, slots):
        row = self.qkv(x)
        n, h, g, d = x.shape[0], self.heads, self.kv_heads, self.dim
        q, k, v = (t.view(n, -1, d) for t in row.split((h * d, g * d, g * d), 1))          # (as they lie in the projection's rows)
        return any4.any4_rope_kv_write(q, k, v, positions, self.freqs, slots.to(self.device), self.cache_k, self.cache_v, self.scales, bits=self.bits,
                                       out=q)                                               # (q is turned where it is)

    def prompt(self, x, tokens):
        before = list(self.lengths)
        slots = torch.cat([self._grow(r, n) for r, n in enumerate(tokens)])
        positions = torch.cat([torch.arange(b, b + n) for b, n in zip(before, tokens)]).to(self.device)
        q = self._project(x, positions, slots)
        starts = torch.tensor([0] + list(tokens), dtype=torch.int32).cumsum(0).to(torch.int32).to(self.device)
        out = any4.any4_attn_chunk(q, self.cache_k, self.cache_v, self.table.to(self.device), starts,
                                   torch.tensor(self.lengths, dtype=torch.int32, device=self.device), self.scales, bits=self.bits, **self.part)
        return self.o(out.view(x.shape[0], -1))

    def token(self, x):
        positions = torch.tensor(self.lengths, device=self.device)
        slots = torch.cat([self._grow(r, 1) for r in range(x.shape[0])])
        q = self._project(x, positions, slots)
        out = any4.any4_attn_decode(q, self.cache_k, self.cache_v, self.table.to(self.device),
                                    torch.tensor(self.lengths, dtype=torch.int32, device=self.device), self.scales, bits=self.bits, **self.part)
        return self.o(out.view(x.shape[0], -1))

    def _sees(self, at):
        ahead = at[:, None] - at
        return (ahead >= 0) & ((ahead < self.part["window"]) | (at < self.part["sinks"]) if self.part else True)


def run(block, requests, prompt, tokens, hidden, seed=0):
    """each request's outputs and inputs, after a prompt in two parts of lengths around `prompt` and `tokens` single tokens"""
    g = torch.Generator().manual_seed(seed)
    lengths = [max(2, prompt - 13 * r) for r in range(requests)]
    x = [(torch.randn(n + tokens, hidden, generator=g) * 0.05).to(torch.bfloat16).to(block.device) for n in lengths]
    got, done = [[] for _ in range(requests)], [0] * requests
    for part in (lambda n: n // 3, lambda n: n - n // 3):
        take = [part(n) for n in lengths]
        y = block.prompt(torch.cat([x[r][done[r]:done[r] + take[r]] for r in range(requests)]), take)
        for r, rows in enumerate(y.split(take)):
            got[r].append(rows)
            done[r] += take[r]
    for _ in range(tokens):
        y = block.token(torch.stack([x[r][done[r]] for r in range(requests)]))
        for r in range(requests):
            got[r].append(y[r:r + 1])
            done[r] += 1
    return [torch.cat(rows) for rows in got], x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, default=8)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--window", type=int)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--separate", action="store_true")
    a = ap.parse_args()
    if a.separate and a.window is not None:
        ap.error("--window goes without --separate")
    if a.sinks and a.window is None:
        ap.error("--sinks go with --window")
    need = -(-(a.prompt + a.tokens) // 64)
    sizes = dict(bits=a.bits, requests=a.requests, max_pages=need, pages=need * a.requests)
    block = AttentionBlock(**sizes) if a.separate else FusedBlock(window=a.window, sinks=a.sinks, **sizes)
    outputs, x = run(block, a.requests, a.prompt, a.tokens, 4096)
    weights = [any4.any4_dequant(w.codes, w.lut, w.scale, w.offset, w.codes.shape[1] * 8, 4) for w in (block.qkv, block.o)]
    for r, y in enumerate(outputs):
        want = block.plain(x[r], weights)
        print(f"request {r}: {y.shape[0]} tokens, cache of {a.bits} bits, relative distance from 32 bits "
              f"{((y.float() - want).norm() / want.norm()).item():.4f}")


if __name__ == "__main__":
    main()
