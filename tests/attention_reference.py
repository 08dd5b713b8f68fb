"""Attention and the cache's number format from their definitions in 64 bits, and how far a 16-bit result may lie from them.

The bound of an output o = sum_j p_j v_j (weights p_j that add to 1), u = 2^-8 for bf16 and 2^-11 for fp16:
  rounding of the result                       u |o|
  rounding of the weights                      u sum_j p_j |v'_j|,  v' the values that the rounded weights multiply (codes: around their centre)
  weights of fp16 below its normal range       2^-25 sum_j |v'_j| / (what the weights add to before they are divided: at least 1)
  scores: dot products of D terms in fp32      2 e sum_j p_j |v_j|, e = 8 sqrt(D) 2^-24 times the products' absolute sum at its largest
                                               (rounding errors of random sign, eight deviations), and exp2's own 2^-20
  sums over n tokens in fp32                   8 sqrt(n) 2^-24 sum_j p_j times the largest value as the matrix cores see it
Codes go through the matrix cores with a bias of up to 1024 on top, which the last two lines count."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def encode(x, bits):
    """fp32 numpy [..., D] -> codes, scale, offset (fp32 that are bf16 values), by the definition in any4.h"""
    x = np.asarray(x, np.float32)
    top = np.float32((1 << bits) - 1)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        scale = bf16((hi - lo) / top)
        offset = bf16(lo)
        broken = ~np.isfinite(x).all(-1, keepdims=True) | ~np.isfinite(scale)
        scale = np.where(scale == 0, np.float32(1), scale)
        codes = np.clip(np.rint((x - offset) / scale), 0, top)
    codes = np.where(broken, 0, codes).astype(np.uint8)
    return codes, np.where(broken, np.float32(np.nan), scale), np.where(broken, np.float32(np.nan), offset)


def bf16(x):
    """fp32 -> nearest bf16, ties to even, as fp32"""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def pack(codes, bits):
    return codes if bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(held, bits):
    if bits == 8:
        return held
    return np.stack((held & 15, held >> 4), -1).reshape(*held.shape[:-1], 2 * held.shape[-1])


def attend(q, k, v, seen, scale):
    """float64 [n, D], [m, D], [m, D], bool [n, m] -> o [n, D]; rows that see nothing are zeros"""
    s = (q @ k.T) * scale
    s = np.where(seen, s, -np.inf)
    top = s.max(1, keepdims=True, initial=-np.inf)
    e = np.where(seen, np.exp(s - np.where(np.isfinite(top), top, 0)), 0)
    total = e.sum(1, keepdims=True)
    p = e / np.where(total == 0, 1, total)
    return p @ np.where(seen.any(0)[:, None], v, 0), p, total


def bound(q, k, v, seen, scale, dtype, bits=16, k_scale=None, v_scale=None, v_offset=None):
    """o and the allowed distance, [n, D] each; k, v finite (float64).  k_scale, v_scale, v_offset: of the tokens, with codes"""
    u = UNIT[dtype]
    D, m = q.shape[1], k.shape[0]
    o, p, total = attend(q, k, v, seen, scale)
    if m == 0:
        return o, np.zeros_like(o)
    bias = 0.0 if bits == 16 else (1024.0 if dtype == torch.float16 else 128.0)
    products = np.abs(q) @ np.abs(k).T
    centred, seen_value = np.abs(v), np.abs(v).max()
    if bits != 16:
        top = (1 << bits) - 1
        products = products + np.abs(q).sum(1, keepdims=True) * (np.abs(k_scale) * (bias + top))[None, :] * 2
        centre = 1 << (bits - 1)
        centred = np.abs(v - (v_offset + centre * v_scale)[:, None])
        seen_value = seen_value + np.abs(v_scale).max() * (bias + top)
    e = 8 * math.sqrt(D) * 2.0 ** -24 * scale * np.where(seen, products, 0).max(1, initial=0.0) + 2.0 ** -20
    small = 2.0 ** -25 * (seen.astype(np.float64) @ centred) / np.maximum(total, 1) if dtype == torch.float16 else 0.0
    sums = 8 * math.sqrt(m) * 2.0 ** -24 * seen_value * p.sum(1)
    allowed = u * np.abs(o) + u * (p @ centred) + small + 2 * e[:, None] * (p @ np.abs(v)) + sums[:, None]
    return o, 1.02 * allowed + 1e-30
