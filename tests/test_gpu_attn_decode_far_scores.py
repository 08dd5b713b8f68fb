"""any4_attn_decode with scores so large that fp32 holds them to more than the exponent's range (2^31 and more, fp16: 2^27), in requests
beside ordinary ones."""
import numpy as np
import pytest
import torch

import attention_close as close
import attention_reference as ref
import paper_2507_04610_amd as any4
from test_gpu_attn_decode_close import cache_of

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("dtype,top,scale", [(BF16, 2e5, None), (BF16, 1e6, None), (BF16, 1e12, 3.0), (F16, 6e4, None), (F16, 6e4, 1.0), (F16, 6e4, 7.3)])
@pytest.mark.parametrize("lengths", [[300, 40, 77], [3000, 129], [50 + i for i in range(40)]])
def test_the_highest_score_takes_all(bits, dim, dtype, top, scale, lengths):
    """one place of q and k holds all of a score; a head's own key is the one whose score lies 2^-9 of its size above the others'"""
    heads, kv_heads = 4, 2
    p = close.Requests(lengths, bits, dtype, dim, heads, kv_heads, seed=13)
    g = torch.Generator().manual_seed(14)
    p.q = torch.zeros_like(p.q)
    p.q[:, :, 5] = (torch.rand(len(lengths), heads, generator=g) * 0.9 + 0.1).mul(top).mul(torch.randint(0, 2, (len(lengths), heads), generator=g) * 2 - 1).to(dtype)
    for k in p.k:
        k.zero_()
        sign = torch.randint(0, 2, k.shape[:2], generator=g) * 2 - 1
        k[:, :, 5] = (torch.rand(k.shape[:2], generator=g) * 0.9 + 0.1).mul(top).mul(sign).to(dtype)
    out = any4.any4_attn_decode(p.q.cuda(), *cache_of(p, 16), bits=bits, softmax_scale=scale).double().cpu().numpy()
    assert np.isfinite(out).all()
    alone = 0
    for i, rows, q, held in p.each():
        score = q @ held.k.T
        for h, row in enumerate(score):
            first, second = np.sort(row)[[-1, -2]]
            if first - second > 2.0 ** -9 * abs(first):
                alone += 1
                want = held.v[row.argmax()]
                assert (np.abs(out[i, rows][h] - want) <= 1.01 * ref.UNIT[dtype] * np.abs(want) + 2.0 ** -20).all()
    assert alone >= len(lengths)
