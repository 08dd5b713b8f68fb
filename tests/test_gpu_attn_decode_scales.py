"""any4_attn_decode over codes whose scales lie far apart, against 64 bits.

The bound has every token with the weight that it has (p_j, adding to 1; v'_j = scale (code - centre), what the rounded weights multiply), u = 2^-8 for bf16, 2^-11 for fp16:
  rounding of the result      u |o|, fp16 below its normal range half of 2^-24
  rounding of the weights     u sum_j p_j |v'_j|; fp16 below its normal range by half of 2^-24 where the largest p_j scale_j is 2^-2 at least, times codes up to the
                              centre: 2^-23 centre n max_j p_j scale_j
  scores                      products of D terms in fp32, eight deviations: e = 8 sqrt(D) 2^-24 scale sum |q| |k'|, k' with the codes' bias of up to 1024; exp2 and its
                              argument 2^-19 (1 + |s| / 16): 2 e sum_j p_j |v_j|
  sums                        8 sqrt(n) 2^-24 sum_j p_j (|v_j| + (bias + 2 centre) scale_j)"""
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
from test_gpu_attn_decode import Problem
from test_gpu_attn_decode_window import seen

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def allowed(q, k, v, scale, dtype, bits, k_scale, v_scale, v_offset):
    centre, D, n, u = 1 << (bits - 1), q.shape[1], len(k), ref.UNIT[dtype]
    o, p, _ = ref.attend(q, k, v, np.ones((len(q), n), bool), scale)
    s = (q @ k.T) * scale
    middle = np.abs(v - (v_offset + centre * v_scale)[:, None])
    products = np.abs(q) @ np.abs(k).T + np.abs(q).sum(1, keepdims=True) * (np.abs(k_scale) * (1024 + 2 * centre))[None]
    e = 8 * math.sqrt(D) * 2.0 ** -24 * scale * np.where(p > 0, products, 0).max(1) + 2.0 ** -19 * (1 + np.abs(s).max(1) / 16)
    weights = u * (p @ middle) + (2.0 ** -23 * centre * n * (p * v_scale).max(1)[:, None] if dtype == F16 else 0.0)
    sums = 8 * math.sqrt(n) * 2.0 ** -24 * (p @ (np.abs(v) + (1024 + 2 * centre) * v_scale[:, None]))
    return o, 1.02 * (u * np.abs(o) + weights + 2 * e[:, None] * (p @ np.abs(v)) + sums) + (2.0 ** -25 if dtype == F16 else 1e-38)


class Scales(Problem):
    def write(self, i, k, v):
        import paper_2507_04610_amd as any4
        t = torch.arange(self.lengths[i])
        slots = (torch.tensor(self.pages_of[i])[t // self.page] * self.page + t % self.page).cuda()
        any4.any4_kv_write(k.to(self.dtype).cuda(), v.to(self.dtype).cuda(), slots, self.ck, self.cv, self.sc, bits=self.bits)

    def near(self, out, window=None, sinks=0):
        out, q, shared = out.double().cpu().numpy(), self.q.double().cpu().numpy(), self.heads // self.kv_heads
        for i, n in enumerate(self.lengths):
            keep = seen(n, window or n, sinks)
            for j in range(self.kv_heads):
                held, rows = [x[keep] for x in self.held(i, j)], slice(j * shared, (j + 1) * shared)
                o, near = allowed(q[i, rows], held[0], held[1], self.dim ** -0.5, self.dtype, self.bits, *held[2:])
                off = np.abs(out[i, rows] - o)
                assert (off <= near).all(), (i, j, np.max(off / near))


LENGTHS = {"short": [300, 77], "cut": [9001, 700]}


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("dtype,ratio", [(F16, 2.0 ** 10), (F16, 2.0 ** 16), (F16, 2.0 ** 20), (BF16, 2.0 ** 20), (BF16, 2.0 ** 60)])
@pytest.mark.parametrize("where", ("first", "middle", "everywhere"))
def test_large_values_of_no_weight(bits, lengths, dim, dtype, ratio, where):
    """tokens whose keys point away from the queries have values far larger than those that carry the weight: their products stay below the others', but their scales do not"""
    p = Scales(LENGTHS[lengths], bits, dtype, dim, 8, 2, 64, seed=51)
    p.q.copy_((p.q * 0.2 + 1).to(dtype))
    for i, n in enumerate(p.lengths):
        g = torch.Generator().manual_seed(i)
        large = {"first": torch.arange(n) < 3, "middle": torch.arange(n) == n // 2, "everywhere": torch.arange(n) % 23 == 5}[where]
        k = torch.randn(n, 2, dim, generator=g) * 0.2 + 1
        k[large] *= -(1.0 + math.log2(ratio) / 10)
        small = 2.0 ** -7 if dtype == F16 else 0.05             # (values up to 6 times 2^13 in fp16)
        p.write(i, k, (torch.randn(n, 2, dim, generator=g) * torch.where(large, small * ratio, small)[:, None, None]).clamp(-6 * small * ratio, 6 * small * ratio))
    p.near(p.run())
    p.near(p.run(window=250, sinks=2), 250, 2)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("dtype", (F16, BF16))
def test_values_that_fall_while_scores_rise(bits, lengths, dtype):
    """scores rise by 30 from the first key to the last while values fall by 2^20, and the other way round"""
    for rising in (True, False):
        p = Scales(LENGTHS[lengths], bits, dtype, 128, 8, 2, 64, seed=52)
        p.q.copy_((p.q * 0.02 + 1).to(dtype))
        for i, n in enumerate(p.lengths):
            g = torch.Generator().manual_seed(i)
            at = torch.linspace(-1, 1, n)[:, None, None] * (1 if rising else -1)
            p.write(i, at * 1.3 + torch.randn(n, 2, 128, generator=g) * 0.02, torch.randn(n, 2, 128, generator=g) * 2.0 ** (-10 * at))
        p.near(p.run())


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("dtype", (F16, BF16))
def test_vectors_of_one_value(bits, lengths, dtype):
    """a constant vector has scale 1 whatever its value: next to values of 1e-3 that is 2^16 times their scale"""
    p = Scales(LENGTHS[lengths], bits, dtype, 128, 8, 2, 64, seed=53)
    p.q.copy_((p.q * 0.2 + 1).to(dtype))
    for i, n in enumerate(p.lengths):
        g = torch.Generator().manual_seed(i)
        k, v = torch.randn(n, 2, 128, generator=g) * 0.2 + 1, torch.randn(n, 2, 128, generator=g) * 1e-3
        alike = torch.arange(n) % 50 == 7
        k[alike] *= -0.7
        v[alike] = torch.tensor([0.0, 3.0, -1e4])[torch.arange(int(alike.sum())) % 3][:, None, None]
        p.write(i, k, v)
    p.near(p.run())
