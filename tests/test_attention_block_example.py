"""examples/attention_block.py: on the CPU with the library's calls replaced by their definitions (pages, slots, positions, parts of a prompt),
on the GPU as it is."""
import importlib.util
import os
import types

import pytest
import torch

import paper_2507_04610_amd as any4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIZES = dict(hidden=256, heads=4, kv_heads=2, head_dim=64, page_size=16, max_pages=8, requests=3, pages=24)


@pytest.fixture()
def example():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def attend(q, k, v, seen):
    k, v = (t.double().repeat_interleave(q.shape[1] // t.shape[1], 1) for t in (k, v))
    out = torch.empty(q.shape, dtype=torch.float64)
    for j in range(q.shape[1]):
        s = (q[:, j].double() @ k[:, j].T) * q.shape[2] ** -0.5
        out[:, j] = torch.softmax(s.masked_fill(~seen, -torch.inf), -1) @ v[:, j]
    return out.to(q.dtype)


def definitions():
    def flat(cache):
        return cache.permute(0, 2, 1, 3).reshape(-1, cache.shape[1], cache.shape[3])

    def kv_write(k, v, slots, ck, cv, scales=None, bits=16):
        page = ck.shape[2]
        ck[slots // page, :, slots % page], cv[slots // page, :, slots % page] = k, v

    def kv_read(ck, cv, slots, scales=None, bits=16, dtype=torch.bfloat16):
        return flat(ck)[slots], flat(cv)[slots]

    def prompt(q, k, v, qs, ks):
        parts = []
        for r in range(len(qs) - 1):
            nq, nk = int(qs[r + 1] - qs[r]), int(ks[r + 1] - ks[r])
            parts.append(attend(q[qs[r]:qs[r + 1]], k[ks[r]:ks[r + 1]], v[ks[r]:ks[r + 1]], torch.ones(nq, nk, dtype=torch.bool).tril(nk - nq)))
        return torch.cat(parts)

    def decode(q, ck, cv, table, lengths, scales=None, bits=16):
        rows = []
        for r, n in enumerate(lengths.tolist()):
            slots = (table[r].long()[:, None] * ck.shape[2] + torch.arange(ck.shape[2])).reshape(-1)[:n]
            rows.append(attend(q[r:r + 1], *kv_read(ck, cv, slots), torch.ones(1, n, dtype=torch.bool)))
        return torch.cat(rows)

    def gemm(x, codes, lut, scale, offset, bits):
        return (x.float() @ weight(codes, lut, scale, offset).T).to(x.dtype)

    def weight(codes, lut, scale, offset):
        w = torch.gather(lut.float(), 1, codes.long())
        return w * scale.float().repeat_interleave(128, 1) + offset.float().repeat_interleave(128, 1)
    return types.SimpleNamespace(any4_pack=lambda codes, bits: codes, any4_gemm=gemm, any4_kv_cache=any4.any4_kv_cache, any4_kv_write=kv_write, any4_kv_read=kv_read,
                                 any4_attn_prompt=prompt, any4_attn_decode=decode), weight


def distance(y, want):
    return ((y.float() - want).norm() / want.norm()).item()


def test_bookkeeping(example, monkeypatch):
    calls, weight = definitions()
    monkeypatch.setattr(example, "any4", calls)
    block = example.AttentionBlock(bits=16, device="cpu", **SIZES)
    outputs, x = example.run(block, 3, 70, 5, 256)
    weights = [weight(w.codes, w.lut, w.scale, w.offset) for w in (block.qkv, block.o)]
    assert block.lengths == [75, 62, 49] and len(block.free) == 24 - 5 - 4 - 4
    for y, rows in zip(outputs, x):
        assert distance(y, block.plain(rows, weights)) < 0.02           # (bf16 between the steps: a few roundings of 2^-9)


@pytest.mark.gpu
@pytest.mark.parametrize("bits,most", [(16, 0.02), (8, 0.03), (4, 0.25)])
def test_block(example, bits, most):
    """8 bits add the rounding to 255 steps of about five deviations (0.6 % of a value), 4 bits to 15 (10 %, in k and in v)"""
    block = example.AttentionBlock(bits=bits, **SIZES)
    outputs, x = example.run(block, 3, 70, 5, 256)
    weights = [any4.any4_dequant(w.codes, w.lut, w.scale, w.offset, w.codes.shape[1] * 8, 4) for w in (block.qkv, block.o)]
    for y, rows in zip(outputs, x):
        assert distance(y, block.plain(rows, weights)) < most
