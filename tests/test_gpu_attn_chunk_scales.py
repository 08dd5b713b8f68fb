"""any4_attn_chunk over codes whose scales lie far apart, against 64 bits.

The bound has every token with the weight that it has (p_j, adding to 1; v'_j = scale (code - centre), what the rounded weights multiply):
  rounding of the result      u |o|, fp16 below its normal range half of 2^-24
  rounding of the weights     2^-11 sum_j p_j |v'_j|: p_j times the scale in fp16, whatever the cache's type; below fp16's normal range by half of 2^-24 where the largest
                              p_j scale_j is 2^-2 at least (2^6 up, and down by exponents rounded up twice and by a tile's scales that are taken as one, which lie within
                              2^3 here or are looked at one by one), times codes up to the centre: 2^-23 centre n max_j p_j scale_j
  scores                      products of D terms in fp32, eight deviations: e = 8 sqrt(D) 2^-24 scale sum |q| |k'|, k' with the codes' bias of up to 1024; exp2 and its
                              argument 2^-19 (1 + |s| / 16): 2 e sum_j p_j |v_j|
  sums                        8 sqrt(n) 2^-24 sum_j p_j (|v_j| + 2 centre scale_j)"""
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
from test_gpu_attn_chunk import Chunks

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def allowed(q, k, v, seen, scale, dtype, bits, k_scale, v_scale, v_offset):
    """o and how far a result may lie from it; q [n, D], k, v [m, D] float64"""
    centre, D = 1 << (bits - 1), q.shape[1]
    o, p, _ = ref.attend(q, k, v, seen, scale)
    s = np.where(seen, (q @ k.T) * scale, 0.0)
    middle = np.abs(v - (v_offset + centre * v_scale)[:, None])
    products = np.abs(q) @ np.abs(k).T + np.abs(q).sum(1, keepdims=True) * (np.abs(k_scale) * (1024 + 2 * centre))[None]
    e = 8 * math.sqrt(D) * 2.0 ** -24 * scale * np.where(seen & (p > 0), products, 0).max(1, initial=0.0) + 2.0 ** -19 * (1 + np.abs(s).max(1) / 16)
    weights = 2.0 ** -11 * (p @ middle) + 2.0 ** -23 * centre * seen.sum(1)[:, None] * (p * v_scale).max(1)[:, None]
    sums = 8 * math.sqrt(len(k)) * 2.0 ** -24 * (p @ (np.abs(v) + 2 * centre * v_scale[:, None]))
    return o, 1.02 * (ref.UNIT[dtype] * np.abs(o) + weights + 2 * e[:, None] * (p @ np.abs(v)) + sums) + (2.0 ** -25 if dtype == F16 else 1e-38)


def check(p, out, requests=None, scale=None, window=None, sinks=0):
    out, q, starts = out.double().cpu().numpy(), p.q.double().cpu().numpy(), p.starts.tolist()
    shared = p.heads // p.kv_heads
    for i in requests if requests is not None else range(len(p.lengths)):
        rows, seen = slice(starts[i], starts[i + 1]), p.seen(i, window, sinks)
        some = seen.any(0)
        for j in range(p.kv_heads):
            held = [x[some] for x in p.held(i, j)]
            for h in range(j * shared, (j + 1) * shared):
                o, near = allowed(q[rows, h], held[0], held[1], seen[:, some], scale or p.dim ** -0.5, p.dtype, p.bits, *held[2:])
                off = np.abs(out[rows, h] - o)
                # (a token with a value beyond its type's range reads back as NaN, and so has who sees it no result)
                assert ((off <= near) | (np.isnan(o) & np.isnan(out[rows, h]))).all(), (i, h, np.max(off / near))


def along(n, kv_heads, dim, g):
    """keys near a direction that the queries are given as well"""
    return torch.randn(n, kv_heads, dim, generator=g) * 0.2 + 1


# 70 rows of 4 heads: tiles of 128 rows; 3 of 4: of 32, cut where the context is long
PARTS = {"wide": [(70, 300)], "narrow": [(3, 400)], "cut": [(3, 5000), (100, 2000)]}


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("dtype,ratio", [(BF16, 2.0 ** 10), (BF16, 2.0 ** 16), (BF16, 2.0 ** 20), (BF16, 2.0 ** 30), (BF16, 2.0 ** 90), (F16, 2.0 ** 10), (F16, 2.0 ** 16), (F16, 2.0 ** 20)])
@pytest.mark.parametrize("where", ("first", "middle", "everywhere"))
def test_large_values_of_no_weight(bits, parts, dtype, ratio, where):
    """tokens whose keys point away from the queries have values far larger than those that carry the weight: their products stay below the others', but their scales do not"""
    p = Chunks(PARTS[parts], bits, dtype, 128, 8, 2, 64, seed=31)
    p.q.copy_((p.q * 0.2 + 1).to(dtype))
    for i, n in enumerate(p.lengths):
        g = torch.Generator().manual_seed(i)
        large = {"first": torch.arange(n) < 3, "middle": torch.arange(n) == n // 2, "everywhere": torch.arange(n) % 23 == 5}[where]
        # (scores of about 11 and -11 k_by: e^-66 and less where the ratio is 2^90)
        k_by = 1.0 + math.log2(ratio) / 15
        k, v = along(n, 2, 128, g), torch.randn(n, 2, 128, generator=g)
        k[large] *= -k_by
        v = v * torch.where(large, 0.05 * ratio, 0.05)[:, None, None] if dtype == BF16 else v * torch.where(large, 2.0 ** -6 * ratio, 2.0 ** -6)[:, None, None].clamp_max(16384)
        p.write(i, k, v)
    check(p, p.run())
    check(p, p.run(window=250, sinks=2), window=250, sinks=2)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("every", (23, 64))
def test_scales_further_apart_than_fp32_reaches(bits, parts, every):
    """values of 1e29 with weights of 2^-270 beside such of 1e-29, from the first token on"""
    p = Chunks(PARTS[parts], bits, BF16, 128, 8, 2, 64, seed=36)
    p.q.copy_((p.q * 0.2 + 1).to(BF16))
    for i, n in enumerate(p.lengths):
        g = torch.Generator().manual_seed(i)
        large = torch.arange(n) % every == 0
        k, v = along(n, 2, 128, g), torch.randn(n, 2, 128, generator=g)
        k[large] *= -16
        p.write(i, k, v * torch.where(large, 1e29, 1e-29)[:, None, None])
    check(p, p.run())


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("parts", PARTS)
def test_large_values_first_then_the_weight(bits, parts):
    """scores rise from the first key to the last by 60 while values fall by 2^40, and the other way round: the largest product moves by little"""
    for rising in (True, False):
        p = Chunks(PARTS[parts], bits, BF16, 128, 8, 2, 64, seed=32)
        p.q.copy_((p.q * 0.02 + 1).to(BF16))
        for i, n in enumerate(p.lengths):
            g = torch.Generator().manual_seed(i)
            at = torch.linspace(-1, 1, n)[:, None, None] * (1 if rising else -1)
            p.write(i, at * 2.5 + torch.randn(n, 2, 128, generator=g) * 0.02, torch.randn(n, 2, 128, generator=g) * 2.0 ** (-20 * at))
        check(p, p.run())


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("parts", PARTS)
def test_vectors_of_one_value(bits, parts):
    """a constant vector has scale 1 whatever its value: next to values of 1e-4 that is 2^20 times their scale, and where it has a weight its products are the largest"""
    p = Chunks(PARTS[parts], bits, BF16, 128, 8, 2, 64, seed=33)
    p.q.copy_((p.q * 0.2 + 1).to(BF16))
    for i, n in enumerate(p.lengths):
        g = torch.Generator().manual_seed(i)
        k, v = along(n, 2, 128, g), torch.randn(n, 2, 128, generator=g) * 1e-4
        alike = torch.arange(n) % 50 == 7
        k[alike] *= -0.7
        v[alike] = torch.tensor([0.0, 3.0, -1e5, 1e34])[torch.arange(int(alike.sum())) % 4][:, None, None]
        v[alike] *= (torch.arange(int(alike.sum())) % 4 < 3)[:, None, None] if i == 0 else 1
        p.write(i, k, v)
    out = p.run()
    assert out.isfinite().all()
    check(p, out)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("q_by,k_by", [(1e-33, 1e33), (1e-35, 1e35), (1e-37, 2e37), (1e33, 1e-33), (1e37, 1e-37)])
def test_small_queries_of_large_keys(bits, parts, q_by, k_by):
    p = Chunks(PARTS[parts], bits, BF16, 128, 8, 2, 64, seed=34, q_by=q_by, k_by=k_by)
    out = p.run()
    assert out.isfinite().all()
    check(p, out)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("q_by,k_by,scale", [(1.0, 1e-35, 3e35), (1e-18, 1e-17, 1e35), (1e20, 1e15, 1e-35), (1e-5, 1e30, 1e-25)])
def test_softmax_scales_of_any_size(bits, parts, q_by, k_by, scale):
    p = Chunks(PARTS[parts], bits, BF16, 128, 8, 2, 64, seed=37, q_by=q_by, k_by=k_by)
    out = p.run(softmax_scale=scale)
    assert out.isfinite().all()
    check(p, out, scale=scale)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype,v_by", [(F16, 1e-3), (F16, 100.0), (BF16, 1e-10), (BF16, 1.0), (BF16, 1e8), (BF16, 1e30)])
@pytest.mark.parametrize("parts", PARTS)
def test_far_scores_that_are_alike(bits, dtype, v_by, parts):
    """one key for all tokens, its score 2^26 (fp16) and 2^33 (bf16): every token that a query sees has the same weight, while v's scales change by 2^12 from tile to tile"""
    p = Chunks(PARTS[parts], bits, dtype, 128, 8, 2, 64, seed=35)
    by = 2.0 ** 12 if dtype == F16 else 2.0 ** 17
    p.q.copy_(torch.full_like(p.q, by / 4))
    for i, n in enumerate(p.lengths):
        g = torch.Generator().manual_seed(i)
        k = torch.full((n, 2, 128), by)
        k[..., ::2] = 0.0                                       # (two values: the codes hold them as they are)
        size = torch.where(torch.arange(n) // 64 % 2 == 0, 1.0, 2.0 ** -12 if dtype == BF16 else 2.0 ** -5)
        p.write(i, k, torch.randn(n, 2, 128, generator=g) * v_by * size[:, None, None])
    out, starts = p.run().double().cpu().numpy(), p.starts.tolist()
    for i in range(len(p.lengths)):
        seen = p.seen(i).astype(np.float64)
        count = seen.sum(1)[:, None]
        for j in range(2):
            _, v, _, vs, vo = p.held(i, j)
            centre = 1 << (bits - 1)
            o = seen @ v / count
            middle = np.abs(v - (vo + centre * vs)[:, None])
            near = ref.UNIT[dtype] * np.abs(o) + 2.0 ** -11 * (seen @ middle) / count + 2.0 ** -23 * centre * vs.max() + 8 * math.sqrt(len(v)) * 2.0 ** -24 * (seen @ (np.abs(v) + 2 * centre * vs[:, None])) / count
            for h in range(4 * j, 4 * j + 4):
                off = np.abs(out[starts[i]:starts[i + 1], h] - o)
                assert (off <= 1.02 * near + 2.0 ** -25 * (dtype == F16)).all(), (i, h, np.max(off / near))
