"""Norm and rotation of heads from their definition in 64 bits, and how far a result in 16 bits may lie from it.

u = 2^-8 for bf16 and 2^-11 for fp16 (half a step, relative), e = 2^-24 (half a step of fp32):
  rounding of the result           u |y|, below fp16's normal range 2^-25
  angle: turns in fp64, what is left of them (at most half a turn, in half turns at most 1) in fp32       pi e
  sine and cosine                  4 steps of fp32 near 1: 8 e
  norm: D squares added in fp32    relative D e in the sum, half of it in the root; the mean, eps, the root, its reciprocal (2 steps each) and two
                                   products: 12 e
  the turn's two products and their sum    3 e
all of them relative to |a| + |b| of the pair (values that are not turned: |y|)."""
import numpy as np

UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
E = 2.0 ** -24


def turn(x, weight, positions, freqs, axis_of=None, interleaved=False, eps=1e-6):
    """x [tokens, heads, D] float64, weight [D] or None, positions int64 [axes, tokens], freqs [rotary / 2] -> y, |a| + |b| of each value's pair"""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * weight
    half = len(freqs)
    axis_of = np.zeros(half, int) if axis_of is None else np.minimum(axis_of, len(positions) - 1)
    angle = positions.astype(np.float64)[axis_of].T * freqs                    # [tokens, half]
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    first = 2 * np.arange(half) if interleaved else np.arange(half)
    second = first + (1 if interleaved else half)
    y, size = x.copy(), np.abs(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    return y, size


def allowed(y, size, dtype):
    name = str(dtype).replace("torch.", "")
    d = y.shape[-1]
    return 1.01 * (UNIT[name] * np.abs(y) + (np.pi + 8 + d / 2 + 12 + 3) * E * size) + (2.0 ** -25 if name == "float16" else 1e-38)
