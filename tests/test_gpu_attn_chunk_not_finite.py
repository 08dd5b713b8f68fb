"""any4_attn_chunk where keys are cut into pieces and values are not finite: who sees such a value has a result that is not finite either, as without pieces, and
nobody else's changes by a bit."""
import numpy as np
import pytest
import torch

from test_gpu_attn_chunk import Chunks

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
NAN = float("nan")
# (new tokens, tokens in front): tiles of 128 rows and of 32, few enough that their keys are cut
PARTS = [[(100, 1900), (3, 2001), (0, 40)], [(130, 19870), (5, 20001)]]


def spoil(p, i, tokens, of, what=NAN):
    """keys' or values' of these tokens of a request; with codes their scales"""
    for t in tokens:
        page, at = p.pages_of[i][t // p.page], t % p.page
        if p.bits == 16:
            (p.ck if of == "k" else p.cv)[page, :, at, 3] = what
        else:
            p.sc[page, :, at, 0 if of == "k" else 2] = what


def is_cut(p):
    from paper_2507_04610_amd import any4_attn_chunk_workspace_bytes
    assert any4_attn_chunk_workspace_bytes(len(p.lengths), len(p.q), p.heads, p.kv_heads, p.dim, p.width * p.page) > 0


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F16, 64)])
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("where", ({}, {"window": 1500, "sinks": 70}))
def test_a_query_that_is_no_number_has_no_result(bits, dtype, dim, parts, where):
    p = Chunks(parts, bits, dtype, dim, 8, 2, 64, seed=21)
    is_cut(p)
    want = p.run(**where)
    rows = [(0, 3), (p.new[0] - 1, 0), (p.new[0] + 1, 7)]
    for at, head in rows:
        p.q[at, head, 17] = NAN
    got = p.run(**where)
    for at, head in rows:
        assert got[at, head].isnan().all(), (at, head)
        got[at, head] = want[at, head]
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("of", ("k", "v"))
@pytest.mark.parametrize("where", ({}, {"window": 700, "sinks": 0}))
def test_first_keys_that_are_no_numbers(bits, of, where):
    """one tile of 64 after the other from the first on, so that at some point they are all that a piece has"""
    p = Chunks(PARTS[0], bits, BF16, 128, 8, 2, 64, seed=22)
    is_cut(p)
    want, starts = p.run(**where).cpu(), p.starts.tolist()
    for tile in range(31):
        for i in range(2):
            spoil(p, i, range(64 * tile, 64 * tile + 64), of)
        got = p.run(**where).cpu()
        for i in range(2):
            touched = torch.from_numpy(p.seen(i, **where)[:, :64 * tile + 64].any(1))
            a, b = got[starts[i]:starts[i + 1]], want[starts[i]:starts[i + 1]]
            assert torch.equal(a[~touched].view(torch.int16), b[~touched].view(torch.int16)), (tile, i)
            assert (~a[touched].isfinite()).flatten(2).any(2).all(), (tile, i)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("parts", PARTS)
def test_a_value_that_is_no_number_counts_however_small_its_weight(bits, parts):
    """the first half's keys point away from the queries, the second half's along them: weights of e^-400 and less"""
    p = Chunks(parts, bits, BF16, 128, 8, 2, 64, seed=23)
    is_cut(p)
    p.q.copy_(p.q.abs() + 1)
    for i, n in enumerate(p.lengths):
        if n > 40:
            g = torch.Generator().manual_seed(i)
            sign = torch.where(torch.arange(n) < n // 2, -8.0, 8.0)[:, None, None]
            p.write(i, (torch.rand(n, 2, 128, generator=g) + 1) * sign, torch.randn(n, 2, 128, generator=g))
    p.check(p.run())
    spoil(p, 0, [5], "v")
    starts = p.starts.tolist()
    got = p.run()
    assert (~got[:starts[1]].isfinite()).flatten(2).any(2).all()
    assert got[starts[1]:].isfinite().all()
