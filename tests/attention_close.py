"""Decode attention's distance from 64 bits as the sum of roundings that are independent of each other, for keys, values and queries of
random sign: what is missing, weighed evenly or counted with a bias that does not go away again lies outside.

With u = 2^-8 for bf16 and 2^-11 for fp16, weights p_j that add to 1, v'_j the values that the rounded weights multiply (codes: around
their centre), one deviation of each part is
  result          u |o| / sqrt(3)                            (half a unit in the last place is at most u; uniform); fp16 below its normal
                                                             range half of 2^-24, as a bound
  weights         u / sqrt(3) (sum p_j^2 v'_j^2)^1/2         and, as far as neighbouring weights round the same way, u |sum p_j v'_j| as a bound
  scores          e (sum p_j^2 (v_j - o)^2)^1/2,             e = scale 2^-24 sqrt(D) times a partial sum of a product of D terms, sqrt(D) rms(q)
                                                             times the largest k (codes: with their bias, times their scale), and 2^-21 (1 + |s|)
  sums            2^-24 (sum over 32 tokens each of (the bias and twice the centre times what their weights times scales add to)^2)^1/2, eight
                  roundings in each, and those of a running sum of n / 32 terms as large as the largest value
A value lies within seven deviations, the bounded parts added; the root of the mean square over all values within one and a half.
fp16 weights below the normal range: 2^-25 sum |v'_j| (codes: |c_j - centre| times the largest scale) over what the weights add to."""
import math

import numpy as np
import torch

import attention_reference as ref

BF16, F16 = torch.bfloat16, torch.float16


class Held:
    """k and v of a request and KV head as a cache of `bits` holds them, [n, D] in float64"""

    def __init__(self, k, v, bits, dtype):
        self.bits, self.dtype = bits, dtype
        if bits == 16:
            self.k, self.v = k.double().numpy(), v.double().numpy()
            return
        kc, ks, ko = (x.astype(np.float64) for x in ref.encode(k.float().numpy(), bits))
        vc, vs, vo = (x.astype(np.float64) for x in ref.encode(v.float().numpy(), bits))
        self.k, self.v = kc * ks + ko, vc * vs + vo
        self.codes, self.k_scale, self.v_scale, self.v_offset = vc, ks, vs, vo


def weigh(q, held, scale, keep=None, even=False):
    """weights [rows, n] that add to 1 and what they add to before that; keep: the tokens that count; even: all the same"""
    s = np.zeros((len(q), len(held.k))) if even else (q @ held.k.T) * scale
    if keep is not None:
        s = np.where(keep, s, -np.inf)
    e = np.exp(s - s.max(1, keepdims=True))
    total = e.sum(1, keepdims=True)
    return e / total, total, np.abs(s[np.isfinite(s)]).max()


def expected(q, held, scale):
    """q [rows, D] float64 -> o, the allowed distance of each value, one deviation of each value (bounded parts included)"""
    (n, D), u, f16 = held.v.shape, ref.UNIT[held.dtype], held.dtype == F16
    p, total, top = weigh(q, held, scale)
    o = p @ held.v
    if held.bits == 16:
        bias = centre = 0
        inner, small = held.v, np.abs(held.v)
        k_top = np.abs(held.k).max()
    else:
        centre = 1 << (held.bits - 1)
        bias = 1024 if f16 else 128 if held.bits == 4 else 0
        inner = held.v - (held.v_offset + centre * held.v_scale)
        small = np.abs(held.codes - centre) * held.v_scale.max()
        k_top = (held.k_scale * (bias + 2 * centre)).max() + np.abs(held.k).max()
    weights = u / math.sqrt(3) * np.sqrt(p ** 2 @ inner ** 2)
    e = scale * 2.0 ** -24 * D * np.sqrt((q ** 2).mean(1, keepdims=True)) * k_top + 2.0 ** -21 * (1 + top)
    scores = e * np.sqrt(np.maximum(p ** 2 @ held.v ** 2 - 2 * o * (p ** 2 @ held.v) + o ** 2 * (p ** 2).sum(1, keepdims=True), 0))
    sums = 2.0 ** -24 * math.sqrt(2 * (n // 32 + 1)) * np.abs(held.v).max() * np.ones_like(o)
    if held.bits != 16:
        w = np.pad(p * held.v_scale[:, 0], ((0, 0), (0, -n % 32))).reshape(len(q), -1, 32).sum(2)
        sums = sums + 2.0 ** -24 * math.sqrt(8) * (bias + 2 * centre) * np.sqrt((w ** 2).sum(1, keepdims=True))
    fixed = u * np.abs(p @ inner) + (2.0 ** -25 * (1 + small.sum(0) / total) if f16 else 0.0)
    allowed = u * np.abs(o) + fixed + 7 * (weights + scores + sums)
    one = np.sqrt(u ** 2 / 3 * o ** 2 + weights ** 2 + scores ** 2 + sums ** 2) + fixed
    return o, allowed, one


def fits(got, q, held, scale):
    """how far [rows, D] lies from 64 bits: the largest share of what a value is allowed, and the mean square's of its own"""
    o, allowed, one = expected(q, held, scale)
    off = got - o
    return float(np.max(np.abs(off) / allowed)), float(np.sqrt((off ** 2).mean() / (one ** 2).mean()) / 1.5)


class Requests:
    """requests of given lengths: q [requests, heads, D], k and v of each, [n, kv_heads, D]"""

    def __init__(self, lengths, bits, dtype, dim, heads, kv_heads, seed, k_by=1.0, v_by=0.5):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.bits, self.dtype, self.dim, self.heads, self.kv_heads = lengths, bits, dtype, dim, heads, kv_heads
        self.q = torch.randn(len(lengths), heads, dim, generator=g).to(dtype)
        self.k, self.v = ([(torch.randn(n, kv_heads, dim, generator=g) * by).to(dtype) for n in lengths] for by in (k_by, v_by))
        self.scale = dim ** -0.5

    def each(self, requests=None):
        """(request, rows of its heads, q, held) of every request and KV head that has tokens"""
        shared = self.heads // self.kv_heads
        for i, n in enumerate(self.lengths):
            if n == 0 or (requests is not None and i not in requests):
                continue
            for j in range(self.kv_heads):
                rows = slice(j * shared, (j + 1) * shared)
                yield i, rows, self.q[i, rows].double().numpy(), Held(self.k[i][:, j], self.v[i][:, j], self.bits, self.dtype)


# What the GPU tests run: name -> (lengths, bits, dtype, dim, heads, kv_heads, seed, k_by, v_by), page size
CASES = {}
for _bits in (16, 8, 4):
    for _dtype, _name in ((BF16, "bf16"), (F16, "fp16")):
        for _dim in (128, 64):
            CASES[f"cut_{_bits}_{_name}_{_dim}"] = ([9001, 0, 5, 4096, 2049], _bits, _dtype, _dim, 4, 1, 1, 1.0, 0.5), 128
        CASES[f"all_blocks_{_bits}_{_name}"] = ([70001], _bits, _dtype, 128, 4, 1, 2, 1.0, 0.5), 64
        for _k, _v in ((5.0, 1.0), (0.5, 300.0), (1.0, 1e-4), (2.0, 0.01)):
            CASES[f"values_{_bits}_{_name}_{_k}_{_v}"] = ([700, 33, 3000], _bits, _dtype, 128, 8, 2, 3, _k, _v), 64
    for _page in (256, 512, 1024):
        CASES[f"page_{_page}_{_bits}"] = ([1300, 1, 1024, 255, 0, 2100], _bits, BF16, 128, 8, 2, 4, 1.0, 0.5), _page
    # 40 query heads on a KV head are three parts of at most 16, 60 requests of them 180 groups: blocks of four wavefronts
    CASES[f"forty_heads_{_bits}"] = ([(53 * i) % 700 for i in range(60)], _bits, BF16, 64, 40, 1, 5, 1.0, 0.5), 32
