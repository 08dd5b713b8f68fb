"""Caches and rows whose bytes lie further apart than 32 bits reach: the same results as from ones that lie together, bit for bit."""
import pytest
import torch

import paper_2507_04610_amd as any4

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
HEADS, KV, DIM, PAGE = 8, 4, 128, 64


def rows(n, heads, seed):
    return torch.randn(n, heads, DIM, generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()


@pytest.mark.parametrize("bits", (16, 8, 4))
def test_pages_behind_4_gib(bits):
    far_pages = (5 << 30) // (KV * PAGE * DIM * bits // 8)
    new, lengths = [40, 3, 200], [700, 2003, 200]
    starts, n = torch.tensor([0, 40, 43, 243], dtype=torch.int32).cuda(), sum(new)
    need = [-(-x // PAGE) for x in lengths]
    order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1))
    length = torch.tensor(lengths, dtype=torch.int32).cuda()
    q, turn = rows(n, HEADS, 2), torch.ones(64, dtype=torch.float64, device="cuda") * 0.01
    got = []
    for pages in (sum(need), far_pages):
        ck, cv, sc = any4.any4_kv_cache(pages, KV, DIM, PAGE, bits)
        if pages == far_pages:
            assert ck.numel() * ck.element_size() > 4 << 30
        table, at = torch.zeros(3, max(need), dtype=torch.int32), 0
        for i, x in enumerate(need):
            table[i, :x] = pages - 1 - order[at:at + x]
            t = torch.arange(lengths[i])
            slots = (table[i, t // PAGE].long() * PAGE + t % PAGE).cuda()
            k, v = rows(lengths[i], KV, 10 + i), rows(lengths[i], KV, 20 + i)
            any4.any4_rope_kv_write(rows(lengths[i], HEADS, 30), k, v, t.cuda(), turn, slots, ck, cv, sc, bits)
            at += x
        table = table.cuda()
        last = q[[39, 42, 242]].contiguous()
        got.append([any4.any4_attn_chunk(q, ck, cv, table, starts, length, sc, bits), any4.any4_attn_chunk(q, ck, cv, table, starts, length, sc, bits, window=150, sinks=7),
                    any4.any4_attn_decode(last, ck, cv, table, length, sc, bits, window=150, sinks=7)])
        del ck, cv, sc
    for a, b in zip(*got):
        assert a.isfinite().all() and torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_rows_behind_4_gib():
    """tokens 8 MiB apart, 600 of them"""
    n, apart = 600, 1 << 22
    q, k, v = rows(n, HEADS, 3), rows(n, KV, 4), rows(n, KV, 5)
    room = torch.zeros(n * apart, dtype=BF16, device="cuda")
    where, turn = torch.arange(n).cuda(), torch.ones(64, dtype=torch.float64, device="cuda") * 0.01
    starts = torch.tensor([0, 250, 600], dtype=torch.int32).cuda()

    def far(x, first):
        y = room.as_strided(x.shape, (apart, DIM, 1), first)
        y.copy_(x)
        return y
    fq, fk, fv = far(q, 0), far(k, 4096), far(v, 8192)
    want = any4.any4_attn_prompt(q, k, v, starts, window=100, sinks=9)
    assert torch.equal(any4.any4_attn_prompt(fq, fk, fv, starts, window=100, sinks=9), want)
    norm = rows(1, 1, 6).view(DIM)
    tq, tk = any4.any4_rope(q, k, where, turn, norm, norm)
    any4.any4_rope(fq, fk, where, turn, norm, norm, out=(fq, fk))
    assert torch.equal(fq, tq) and torch.equal(fk, tk)
    ck, cv, _ = any4.any4_kv_cache(16, KV, DIM, PAGE)
    table, length = torch.arange(16, dtype=torch.int32).view(2, 8).cuda(), torch.tensor([250, 350], dtype=torch.int32).cuda()
    slots = torch.cat((torch.arange(250), 512 + torch.arange(350))).cuda()
    near = any4.any4_rope_kv_write(fq, fk, fv, where, turn, slots, ck, cv)
    again = [x.clone() for x in (ck, cv)]
    assert torch.equal(near, any4.any4_rope_kv_write(tq, tk, v, where, turn, slots, ck, cv)) and torch.equal(ck, again[0]) and torch.equal(cv, again[1])
    assert torch.equal(any4.any4_attn_chunk(fq, ck, cv, table, starts, length), any4.any4_attn_chunk(tq, ck, cv, table, starts, length))
