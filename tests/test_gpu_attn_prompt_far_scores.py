"""any4_attn_prompt with scores so large that fp32 holds them to more than the exponent's range (2^31 and more, fp16: 2^27), beside rows
of ordinary ones."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2507_04610_amd as any4

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("dtype,top,scale", [(BF16, 2e5, None), (BF16, 1e6, None), (BF16, 1e12, 3.0), (F16, 6e4, None), (F16, 6e4, 1.0), (F16, 6e4, 7.3)])
@pytest.mark.parametrize("n,ahead,causal", [(300, 0, True), (130, 411, True), (257, 0, False)])
def test_the_highest_score_takes_all(dtype, top, scale, dim, n, ahead, causal):
    """one place of q and k holds all of a score: query i times key j, products of two short numbers, apart by 2^-8 of their size at least
    where they differ at all"""
    g = torch.Generator().manual_seed(int(n + dim))
    m = n + ahead
    heads = 2
    # keys of both signs, no two alike: 2^-7 of their size apart in bf16, 2^-10 in fp16
    size = torch.unique((torch.rand(40 * m, generator=g) * 0.9 + 0.1).mul(top).to(dtype)).double()
    size = size[torch.randperm(len(size), generator=g)]
    keys = torch.cat((size, -size, size / 16, -size / 16, size / 256, -size / 256)).to(dtype).unique()
    keys = keys[torch.randperm(len(keys), generator=g)][:m]
    m = len(keys)
    n = m - ahead
    assert n > 100
    at = torch.rand(n, heads, generator=g).mul(0.9).add(0.1).mul(top).mul(torch.randint(0, 2, (n, heads), generator=g) * 2 - 1).to(dtype)
    near = torch.arange(n) % 7 == 3                                       # every seventh query has ordinary scores
    s = dim ** -0.5 if scale is None else scale
    at[near] = (torch.randn(int(near.sum()), heads, generator=g) * (4.0 / s / top)).to(dtype)
    q, k = torch.zeros(n, heads, dim, dtype=dtype), torch.zeros(m, 1, dim, dtype=dtype)
    q[:, :, 5], k[:, 0, 5] = at, keys
    v = torch.randn(m, 1, dim, generator=g).to(dtype)
    starts = [torch.tensor([0, x], dtype=torch.int32).cuda() for x in (n, m)]
    out = any4.any4_attn_prompt(q.cuda(), k.cuda(), v.cuda(), *starts, causal=causal, softmax_scale=scale).cpu()
    seen = np.tril(np.ones((n, m), bool), m - n) if causal else np.ones((n, m), bool)
    for h in range(heads):
        score = np.where(seen, np.outer(at[:, h].double().numpy(), keys.double().numpy()), -np.inf)
        best = np.sort(score, 1)[:, -2:]
        alone = ~near.numpy() & (best[:, 1] - best[:, 0] > 2.0 ** -9 * np.abs(best[:, 1]).clip(1e8 / s)) | (seen.sum(1) == 1)
        assert alone.sum() > n // 3
        rows = torch.from_numpy(np.flatnonzero(alone))
        assert torch.equal(out[rows, h], v[torch.from_numpy(score.argmax(1)[alone]), 0])
        rows = np.flatnonzero(near.numpy())
        o, allowed = ref.bound(q[rows, h].double().numpy(), k[:, 0].double().numpy(), v[:, 0].double().numpy(), seen[rows], s, dtype)
        assert (np.abs(out[rows, h].double().numpy() - o) <= allowed).all()
    assert out.isfinite().all()
