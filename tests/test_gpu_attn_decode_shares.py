"""any4_attn_decode with many requests: blocks of 4 wavefronts (from 64 groups of request and KV head on), more requests than a wavefront
has lanes, more than one launch takes."""
import pytest
import torch

import paper_2507_04610_amd as any4
from test_gpu_attn_decode import BF16, F16, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
def test_blocks_of_four_wavefronts(bits, dtype, dim):
    lengths = [0, 1, 31, 32, 33, 127, 128, 129, 255, 257, 2000] + [(37 * i) % 300 for i in range(29)]
    p = Problem(lengths, bits, dtype, dim, 8, 2, 32, seed=20 + bits)
    out = p.run()
    p.check(out)
    assert torch.equal(out.view(torch.int16), p.run().view(torch.int16))


@pytest.mark.parametrize("bits", (16, 8, 4))
def test_more_requests_than_lanes(bits):
    lengths = [(53 * i) % 190 for i in range(150)]
    lengths[70] = 3000
    p = Problem(lengths, bits, BF16, 64, 2, 1, 16, seed=30)
    p.check(p.run())


def test_full_wavefront_of_requests():
    p = Problem([700 + 11 * i for i in range(64)], 8, BF16, 128, 4, 1, 64, seed=31)
    p.check(p.run())


@pytest.mark.parametrize("bits", (16, 4))
def test_one_request_on_all_blocks(bits):
    """as many pieces to join as there are blocks: more than a wavefront has lanes"""
    p = Problem([70001], bits, BF16, 128, 4, 1, 64, seed=33)
    out = p.run()
    p.check(out)
    assert torch.equal(out.view(torch.int16), p.run().view(torch.int16))


def test_more_requests_than_a_launch_takes():
    """2500 requests over the pages of one: their own lengths, the same results as in calls of a few"""
    p = Problem([200], 16, BF16, 64, 2, 1, 16, seed=32)
    n = 2500
    lengths = (torch.arange(n) * 7 % 201).to(torch.int32).cuda()
    q = torch.randn(n, 2, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    table = p.table.expand(n, -1).contiguous()
    out = any4.any4_attn_decode(q, p.ck, p.cv, table, lengths)
    for at in (0, 1000, 2040, 2490):
        few = any4.any4_attn_decode(q[at:at + 10], p.ck, p.cv, table[at:at + 10], lengths[at:at + 10].clone())
        assert (out[at:at + 10].float() - few.float()).abs().max() <= 2.0 ** -5          # (two roundings each of sums and weights of up to 2)
    assert not out[lengths == 0].any()
