"""The fused block of examples/attention_block.py (rotation and cache write in one call, attention of prompts' parts and single tokens over the pages):
on the CPU with the library's calls replaced by their definitions, on the GPU as it is, and there the same bits from captured and replayed calls."""
import importlib.util
import os
import types

import pytest
import torch

import paper_2507_04610_amd as any4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIZES = dict(hidden=256, heads=4, kv_heads=2, head_dim=64, page_size=16, max_pages=8, requests=3, pages=24)
PARTS = [dict(), dict(window=20), dict(window=33, sinks=3)]


@pytest.fixture()
def example():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def definitions():
    def turn(x, positions, freqs):
        half = freqs.numel()
        angle = (positions[:, None].double() * freqs)[:, None]
        a, b = x[..., :half].double(), x[..., half:].double()
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1).to(x.dtype)

    def rope_kv_write(q, k, v, positions, freqs, slots, ck, cv, scales=None, bits=16, out=None):
        page = ck.shape[2]
        ck[slots // page, :, slots % page], cv[slots // page, :, slots % page] = turn(k, positions, freqs), v
        out.copy_(turn(q, positions, freqs))
        return out

    def chunk(q, ck, cv, table, starts, lengths, scales=None, bits=16, window=None, sinks=0):
        page, out = ck.shape[2], torch.empty(q.shape, dtype=q.dtype)
        for r, n in enumerate(lengths.tolist()):
            at = table[r].long().repeat_interleave(page)[:n], torch.arange(n) % page
            k, v = (c[at[0], :, at[1]].double() for c in (ck, cv))
            lo, hi = int(starts[r]), int(starts[r + 1])
            p, j = torch.arange(n - hi + lo, n)[:, None], torch.arange(n)
            seen = (j <= p) & ((j > p - window) | (j < sinks)) if window is not None else j <= p
            for h in range(q.shape[1]):
                g = h // (q.shape[1] // ck.shape[1])
                s = (q[lo:hi, h].double() @ k[:, g].T) * q.shape[2] ** -0.5
                out[lo:hi, h] = (torch.softmax(s.masked_fill(~seen, -torch.inf), -1) @ v[:, g]).to(q.dtype)
        return out

    def decode(q, ck, cv, table, lengths, scales=None, bits=16, window=None, sinks=0):
        return chunk(q, ck, cv, table, torch.arange(q.shape[0] + 1), lengths, window=window, sinks=sinks)

    def weight(codes, lut, scale, offset):
        return torch.gather(lut.float(), 1, codes.long()) * scale.float().repeat_interleave(128, 1) + offset.float().repeat_interleave(128, 1)

    def gemm(x, codes, lut, scale, offset, bits):
        return (x.float() @ weight(codes, lut, scale, offset).T).to(x.dtype)
    return types.SimpleNamespace(any4_pack=lambda codes, bits: codes, any4_gemm=gemm, any4_kv_cache=any4.any4_kv_cache,
                                 any4_rope_kv_write=rope_kv_write, any4_attn_chunk=chunk, any4_attn_decode=decode), weight


def distance(y, want):
    return ((y.float() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("part", PARTS)
def test_bookkeeping(example, monkeypatch, part):
    calls, weight = definitions()
    monkeypatch.setattr(example, "any4", calls)
    block = example.FusedBlock(bits=16, device="cpu", **part, **SIZES)
    outputs, x = example.run(block, 3, 70, 5, 256)
    weights = [weight(w.codes, w.lut, w.scale, w.offset) for w in (block.qkv, block.o)]
    assert block.lengths == [75, 62, 49] and len(block.free) == 24 - 5 - 4 - 4
    for y, rows in zip(outputs, x):
        assert distance(y, block.plain(rows, weights)) < 0.02           # (bf16 between the steps: a few roundings of 2^-9)


@pytest.mark.gpu
@pytest.mark.parametrize("part", PARTS)
@pytest.mark.parametrize("bits,most", [(16, 0.02), (8, 0.03), (4, 0.25)])
def test_block(example, bits, most, part):
    """8 bits add the rounding to 255 steps of about five deviations (0.6 % of a value), 4 bits to 15 (10 %, in k and in v)"""
    block = example.FusedBlock(bits=bits, **part, **SIZES)
    outputs, x = example.run(block, 3, 70, 5, 256)
    weights = [any4.any4_dequant(w.codes, w.lut, w.scale, w.offset, w.codes.shape[1] * 8, 4) for w in (block.qkv, block.o)]
    for y, rows in zip(outputs, x):
        assert distance(y, block.plain(rows, weights)) < most


@pytest.mark.gpu
@pytest.mark.parametrize("bits", (16, 8, 4))
def test_captured_steps(example, bits):
    """A graph of a layer's drafts (rotation and write, attention of 4 tokens a request) and then of one token (both calls again) holds two steps of
    serving; replayed with lengths, slots and rows changed in place, and eager calls between, it gives the bits of eager calls on a cache of its own."""
    page, requests, width, heads, kv_heads, dim = 16, 3, 8, 4, 2, 64
    g = torch.Generator().manual_seed(bits)
    table = torch.randperm(requests * width, generator=g).to(torch.int32).view(requests, width)
    freqs = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64) / (dim // 2)).cuda()
    caches = [any4.any4_kv_cache(requests * width, kv_heads, dim, page, bits, device="cuda") for _ in range(2)]
    on = table.cuda()
    starts, counts = torch.tensor([0, 4, 4, 7], dtype=torch.int32).cuda(), [4, 0, 3]

    def where(lengths, tokens):
        at = [torch.arange(n - t, n) for n, t in zip(lengths, tokens)]
        return torch.cat(at), torch.cat([table[r].long()[p // page] * page + p % page for r, p in enumerate(at)])

    def inputs(lengths):
        after = [n + 1 for n in lengths]
        return [t.cuda() for t in (torch.randn(7, (heads + 2 * kv_heads) * dim, generator=g).to(torch.bfloat16), *where(lengths, counts),
                                   torch.tensor(lengths, dtype=torch.int32), torch.randn(3, (heads + 2 * kv_heads) * dim, generator=g).to(torch.bfloat16),
                                   *where(after, [1] * requests), torch.tensor(after, dtype=torch.int32))]

    def step(cache, rows, at, slots, lengths, row, at1, slots1, after):
        ck, cv, scales = cache
        split = lambda t: [s.view(t.shape[0], -1, dim) for s in t.split((heads * dim, kv_heads * dim, kv_heads * dim), 1)]      # noqa: E731
        q = any4.any4_rope_kv_write(*split(rows), at, freqs, slots, ck, cv, scales, bits=bits)
        drafts = any4.any4_attn_chunk(q, ck, cv, on, starts, lengths, scales, bits=bits, window=40, sinks=2)
        q = any4.any4_rope_kv_write(*split(row), at1, freqs, slots1, ck, cv, scales, bits=bits)
        return drafts, any4.any4_attn_decode(q, ck, cv, on, after, scales, bits=bits, window=40, sinks=2)

    for cache in caches:                                                # a context of noise in both caches
        n = requests * width * page
        k, v = (torch.randn(n, kv_heads, dim, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (1, 2))
        any4.any4_kv_write(k, v, torch.arange(n).cuda(), *cache, bits=bits)
    held = inputs([60, 5, 90])
    step(caches[0], *held), step(caches[1], *held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0], *held)
    for lengths in ([64, 1, 97], [4, 17, 3], [127, 40, 64], [64, 1, 97]):
        for to, new in zip(held, inputs(lengths)):
            to.copy_(new)
        graph.replay()
        want = step(caches[1], *held)
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want)), lengths
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*caches) if a is not None), lengths
