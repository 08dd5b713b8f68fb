"""The cache's and the prompts' calls where one launch does not take all blocks (2^32 threads and more)."""
import pytest
import torch

import paper_2507_04610_amd as any4

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.mark.parametrize("dim,limit", [(128, 2 ** 28), (64, 2 ** 29)])
def test_write_of_more_tokens_than_a_launch_takes(dim, limit):
    """nearly all of them without a slot; the same k and v for all (strides of 0)"""
    n = limit + 70
    k, v = (torch.randn(1, 1, dim, generator=torch.Generator().manual_seed(s)).to(BF16).cuda() for s in (1, 2))
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    at = [0, 1, limit - 17, limit - 16, limit - 15, limit - 1, limit, limit + 1, n - 1]
    ck, cv, _ = any4.any4_kv_cache(2, 1, dim, 16)
    slots[at] = torch.arange(3, 3 + len(at), device="cuda")
    any4.any4_kv_write(k.expand(n, 1, dim), v.expand(n, 1, dim), slots, ck, cv)
    for cache, row in ((ck, k), (cv, v)):
        rows = cache.view(32, dim)
        assert torch.equal(rows[3:3 + len(at)], row.view(1, dim).expand(len(at), dim))
        assert not rows[:3].any() and not rows[3 + len(at):].any()


def test_prompt_of_more_blocks_than_a_launch_takes():
    """600 requests of one token each, 32768 query heads: 19.8 million blocks; one key each, so the output is its v"""
    n, heads, dim = 600, 32768, 64
    g = torch.Generator().manual_seed(3)
    q = torch.randn(1, heads, dim, generator=g).to(BF16).cuda().expand(n, heads, dim)
    k, v = (torch.randn(n, 1, dim, generator=g).to(BF16).cuda() for _ in range(2))
    out = any4.any4_attn_prompt(q, k, v, torch.arange(n + 1, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, v.expand(n, heads, dim))
