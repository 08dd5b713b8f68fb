"""any4_attn_decode against 64 bits under the narrow bound of attention_close.py (which a missing piece or even weights exceed, see
test_attention_close.py), and with more tokens in one block's sums than a bias on the codes would survive."""
import pytest
import torch

import attention_close as close
import paper_2507_04610_amd as any4

pytestmark = pytest.mark.gpu


def cache_of(p, page, seed=0):
    """the requests' tokens in a cache in pages of any order: what a decode call takes behind q"""
    need = [-(-n // page) for n in p.lengths]
    order = torch.randperm(sum(need) + 1, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    ck, cv, scales = any4.any4_kv_cache(len(order), p.kv_heads, p.dim, page, p.bits, p.dtype)
    table, at = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
        if p.lengths[i]:
            t = torch.arange(p.lengths[i])
            slots = (table[i].long()[t // page] * page + t % page).cuda()
            any4.any4_kv_write(p.k[i].cuda(), p.v[i].cuda(), slots, ck, cv, scales, bits=p.bits)
    return ck, cv, table.cuda(), torch.tensor(p.lengths, dtype=torch.int32).cuda(), scales


def check(p, out, requests=None):
    out = out.double().cpu().numpy()
    for i, rows, q, held in p.each(requests):
        worst, mean = close.fits(out[i, rows], q, held, p.scale)
        assert worst <= 1 and mean <= 1, (i, rows, worst, mean)
    for i, n in enumerate(p.lengths):
        assert n or not out[i].any()


@pytest.mark.parametrize("name", close.CASES)
def test_close_to_64_bits(name):
    args, page = close.CASES[name]
    p = close.Requests(*args)
    out = any4.any4_attn_decode(p.q.cuda(), *cache_of(p, page), bits=p.bits)
    check(p, out)


@pytest.mark.parametrize("bits,dtype", [(4, close.F16), (8, close.F16), (4, close.BF16), (8, close.BF16), (16, close.F16)])
@pytest.mark.parametrize("dim", (128, 64))
def test_long_requests_that_are_not_cut(bits, dtype, dim):
    """1024 requests of 131072 tokens each (the same ones): more requests than blocks, each block adds up whole requests"""
    n, requests, page = 131072, 1024, 128
    p = close.Requests([n], bits, dtype, dim, 4, 1, seed=8)
    ck, cv, table, length, scales = cache_of(p, page)
    p.q = torch.randn(requests, 4, dim, generator=torch.Generator().manual_seed(9)).to(dtype)
    out = any4.any4_attn_decode(p.q.cuda(), ck, cv, table.expand(requests, -1).contiguous(), length.expand(requests).contiguous(), scales, bits=bits)
    out = out.double().cpu().numpy()
    held = close.Held(p.k[0][:, 0], p.v[0][:, 0], bits, dtype)
    for i in (0, 1, 500, 1023):
        worst, mean = close.fits(out[i], p.q[i].double().numpy(), held, p.scale)
        assert worst <= 1 and mean <= 1, (i, worst, mean)


def test_requests_of_the_second_launch():
    """2048 requests are one launch: those behind them lie as close as those in front"""
    p = close.Requests([200], 16, close.BF16, 64, 2, 1, seed=10)
    ck, cv, table, _, _ = cache_of(p, 16)
    n = 2500
    lengths = torch.arange(n) * 7 % 201
    q = torch.randn(n, 2, 64, generator=torch.Generator().manual_seed(11)).to(close.BF16)
    out = any4.any4_attn_decode(q.cuda(), ck, cv, table.expand(n, -1).contiguous(), lengths.to(torch.int32).cuda()).double().cpu().numpy()
    for i in (1, 1000, 2046, 2047, 2048, 2049, 2200, 2499):
        m = int(lengths[i])
        held = close.Held(p.k[0][:m, 0], p.v[0][:m, 0], 16, close.BF16)
        worst, mean = close.fits(out[i], q[i].double().numpy(), held, p.scale)
        assert worst <= 1 and mean <= 1, (i, m, worst, mean)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("heads", (1, 3, 5))
@pytest.mark.parametrize("lengths", [[700], [1300], [2900, 1000], [260, 9000]])
def test_odd_numbers_of_heads_and_pieces(bits, heads, lengths):
    """the join's sums lie behind as many factors as there are heads and pieces"""
    p = close.Requests(lengths, bits, close.BF16, 128, heads, 1, seed=12)
    check(p, any4.any4_attn_decode(p.q.cuda(), *cache_of(p, 64), bits=bits))
