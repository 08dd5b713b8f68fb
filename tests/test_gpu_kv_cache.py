"""any4_kv_write / any4_kv_read against the definition in numpy: codes, scales and offsets bit for bit, what is read back bit for bit
(one fp32 fma, rounded once), nothing else touched."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2507_04610_amd as any4

pytestmark = pytest.mark.gpu


def bits_of(t):
    return t.contiguous().view(torch.uint8).cpu()


def rows(n, heads, dim, dtype, seed, fused):
    """k, v [n, heads, dim]; fused: slices of rows that hold other things too"""
    g = torch.Generator().manual_seed(seed)
    if fused:
        row = torch.randn(n, (5 + 2 * heads) * dim, generator=g).to(dtype).cuda()
        return row[:, 5 * dim:(5 + heads) * dim].view(n, heads, dim), row[:, (5 + heads) * dim:].view(n, heads, dim)
    k, v = (torch.randn(heads, n, dim, generator=g).to(dtype).cuda().transpose(0, 1) for _ in range(2))      # head-major
    return k, v


def filled(pages, heads, dim, page, bits, dtype):
    ck, cv, sc = any4.any4_kv_cache(pages, heads, dim, page, bits, dtype)
    for t in (ck, cv, sc):
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)
    return ck, cv, sc


def check_written(k, v, slots, ck, cv, sc, bits, page, touched):
    """every slot of the cache: what was written into it, or what was there before"""
    for which, (x, cache) in enumerate(((k, ck), (v, cv))):
        held = cache.permute(0, 2, 1, 3).reshape(-1, cache.shape[1], cache.shape[3]).cpu()
        if bits == 16:
            want = x.cpu()
        else:
            codes, scale, offset = ref.encode(x.float().cpu().numpy(), bits)
            want = torch.from_numpy(ref.pack(codes, bits))
            so = sc.permute(0, 2, 1, 3).reshape(-1, sc.shape[1], 4)[:, :, 2 * which:2 * which + 2].float().cpu().numpy()
            assert np.array_equal(so[slots[touched]], np.concatenate((scale, offset), -1)[touched], equal_nan=True)
        assert torch.equal(bits_of(held[slots[touched]]), bits_of(want[touched]))
        rest = np.ones(held.shape[0], bool)
        rest[slots[touched]] = False
        assert (bits_of(held[torch.from_numpy(rest)]) == 0x5A).all()
    if bits != 16:
        rest = np.ones(sc.shape[0] * page, bool)
        rest[slots[touched]] = False
        left = sc.permute(0, 2, 1, 3).reshape(-1, sc.shape[1], 4)[torch.from_numpy(rest).cuda()]
        assert (bits_of(left) == 0x5A).all()


def check_read(ck, cv, sc, slots, bits, dtype, page):
    k, v = any4.any4_kv_read(ck, cv, torch.from_numpy(slots).cuda(), sc, bits=bits, dtype=dtype)
    total = ck.shape[0] * page
    inside = (slots >= 0) & (slots < total)
    for which, (got, cache) in enumerate(((k, ck), (v, cv))):
        held = cache.permute(0, 2, 1, 3).reshape(total, cache.shape[1], cache.shape[3]).cpu()[slots[inside]]
        if bits == 16:
            want = held
        else:
            so = sc.permute(0, 2, 1, 3).reshape(total, sc.shape[1], 4)[:, :, 2 * which:2 * which + 2].double().cpu()[slots[inside]]
            c = torch.from_numpy(ref.unpack(held.numpy(), bits)).double()
            want = (c * so[..., :1] + so[..., 1:]).float()                     # (exact in 64 bits, then one fp32 rounding)
            want = (want if dtype == torch.bfloat16 else want.clamp(-65504, 65504)).to(dtype)
        got = got.cpu()
        assert torch.equal(got[torch.from_numpy(inside)].view(torch.int16)[~want.isnan()], want.view(torch.int16)[~want.isnan()])
        assert torch.equal(got[torch.from_numpy(inside)].isnan(), want.isnan())
        assert (got[torch.from_numpy(~inside)].view(torch.int16) == 0).all()


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("heads,dim,page,tokens,fused", [(1, 128, 16, 1, True), (3, 64, 32, 37, False), (8, 128, 64, 200, True), (2, 64, 1024, 513, True),
                                                         (5, 128, 128, 16, False), (1, 64, 16, 33, True)])
def test_write_and_read(bits, dtype, heads, dim, page, tokens, fused):
    pages = -(-tokens // page) + 2
    k, v = rows(tokens, heads, dim, dtype, seed=tokens + bits, fused=fused)
    ck, cv, sc = filled(pages, heads, dim, page, bits, dtype)
    slots = np.random.default_rng(tokens).permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 3:
        slots[1], slots[tokens - 1] = -1, pages * page                          # padding, and one past the end
    touched = (slots >= 0) & (slots < pages * page)
    any4.any4_kv_write(k, v, torch.from_numpy(slots).cuda(), ck, cv, sc, bits=bits)
    check_written(k, v, slots, ck, cv, sc, bits, page, touched)
    wanted = np.concatenate((slots[::-1], slots[:5], [-7, 1 << 40])).astype(np.int64)     # any order, repeats, none
    check_read(ck, cv, sc, wanted, bits, dtype, page)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("dim", (64, 128))
def test_values_that_are_hard_to_hold(bits, dtype, dim):
    """constants, zeros of both signs, one outlier, ties, subnormals, the type's extremes, what is not finite"""
    top = torch.finfo(dtype).max
    g = torch.Generator().manual_seed(3)
    x = torch.randn(16, 1, dim, generator=g)
    x[0], x[1], x[2] = 0.0, -0.0, 3.25
    x[3, 0, 7] = 1000.0
    x[4, 0] = torch.arange(dim) % 16 * 0.5                                       # grid values and halves between them
    x[4, 0, 0], x[4, 0, 1] = 0.0, (1 << bits) - 1.0
    x[5] *= torch.finfo(dtype).tiny
    x[6] *= torch.finfo(dtype).tiny / 64
    x[7, 0, 3], x[7, 0, 4] = top, -top
    x[8, 0, 5] = float("nan")
    x[9, 0, 0] = float("inf")
    x[10, 0, dim - 1] = -float("inf")
    x[11] = float("nan")
    x[12, 0] = torch.where(torch.arange(dim) % 2 == 0, 1.0, -1.0)
    x[13] = -5.0 - x[13].abs()
    x[14] = 100.0 + x[14]
    x = x.to(dtype).cuda()
    ck, cv, sc = filled(3, 1, dim, 16, bits, dtype)
    slots = np.arange(16, dtype=np.int64) + 11
    any4.any4_kv_write(x, x.flip(0), torch.from_numpy(slots).cuda(), ck, cv, sc, bits=bits)
    check_written(x, x.flip(0), slots, ck, cv, sc, bits, 16, np.ones(16, bool))
    check_read(ck, cv, sc, slots, bits, dtype, 16)
    k, _ = any4.any4_kv_read(ck, cv, torch.from_numpy(slots).cuda(), sc, bits=bits, dtype=dtype)
    broken = ~x.isfinite().all(-1)
    if dtype == torch.bfloat16:
        broken[7] = True                                                         # (its range is no fp32 number)
    assert k[broken].isnan().all() and k[~broken].isfinite().all()


@pytest.mark.parametrize("bits", (16, 8, 4))
def test_slots_past_four_gigabytes(bits):
    heads, dim, page = 8, 128, 128
    per_page = heads * page * dim * bits // 8
    pages = (5 << 30) // per_page
    ck, cv = (torch.empty((pages, heads, page, dim * bits // 8 if bits < 16 else dim), dtype=torch.uint8 if bits < 16 else torch.bfloat16, device="cuda")
              for _ in range(2))
    sc = None if bits == 16 else torch.empty((pages, heads, page, 4), dtype=torch.bfloat16, device="cuda")
    k, v = rows(40, heads, dim, torch.bfloat16, 1, True)
    slots = torch.arange(40, device="cuda") + pages * page - 45
    any4.any4_kv_write(k, v, slots, ck, cv, sc, bits=bits)
    for which, (x, cache) in enumerate(((k, ck), (v, cv))):
        held = cache[-1].permute(1, 0, 2)[page - 45:page - 5]
        want = x if bits == 16 else torch.from_numpy(ref.pack(ref.encode(x.float().cpu().numpy(), bits)[0], bits)).cuda()
        assert torch.equal(held, want)
    got = any4.any4_kv_read(ck, cv, slots, sc, bits=bits)
    assert got[0].isfinite().all() and (got[0] - k).abs().max() <= (0 if bits == 16 else 1.0) and (got[1] - v).abs().max() <= (0 if bits == 16 else 1.0)


def test_empty_calls_streams_and_graphs():
    ck, cv, sc = any4.any4_kv_cache(4, 2, 128, 16, bits=8)
    none = torch.empty(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    any4.any4_kv_write(none, none, torch.empty(0, dtype=torch.int64, device="cuda"), ck, cv, sc, bits=8)
    k, v = any4.any4_kv_read(ck, cv, torch.empty(0, dtype=torch.int64, device="cuda"), sc, bits=8)
    assert k.shape == v.shape == (0, 2, 128) and not ck.any()
    x, y = rows(20, 2, 128, torch.bfloat16, 5, True)
    x2, y2 = x.clone(), y.clone()
    slots = torch.arange(20, device="cuda")
    out = tuple(torch.empty(20, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        any4.any4_kv_write(x2, y2, slots, ck, cv, sc, bits=8)
        any4.any4_kv_read(ck, cv, slots, sc, bits=8, out=out)
        side.synchronize()
        want = [t.clone() for t in out]
        with torch.cuda.graph(graph, stream=side):
            any4.any4_kv_write(x2, y2, slots, ck, cv, sc, bits=8)
            any4.any4_kv_read(ck, cv, slots, sc, bits=8, out=out)
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(3):
        x2.copy_(x * (turn + 1))
        graph.replay()
        torch.cuda.synchronize()
        any4.any4_kv_write(x * (turn + 1), y2, slots, ck, cv, sc, bits=8)
        eager = any4.any4_kv_read(ck, cv, slots, sc, bits=8)
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])
    assert torch.equal(want[1], out[1])


def test_refusals_name_the_mistake():
    ck, cv, sc = any4.any4_kv_cache(4, 2, 128, 16, bits=4)
    k, v = rows(6, 2, 128, torch.bfloat16, 5, True)
    slots = torch.arange(6, device="cuda")
    for args, words in (((k.half(), v, slots, ck, cv, sc, 4), "v must have dtype"), ((k, v, slots.int(), ck, cv, sc, 4), "slots must have dtype"),
                        ((k, v, slots[:5], ck, cv, sc, 4), "k must have shape"), ((k, v, slots, ck, cv, None, 4), "scales must be"),
                        ((k, v, slots, ck, cv, sc[:3], 4), "scales must have shape"), ((k, v, slots, ck, cv[:, :1], sc, 4), "cache_v must"),
                        ((k, v, slots, ck, cv, sc, 8), "k must have shape"), ((k, v, slots, ck, cv, None, 16), "cache_k must have dtype"),
                        ((k[:, :, ::2], v, slots, ck, cv, sc, 4), "k must have shape"), ((k, v, slots, ck, cv, sc, 2), "bits must be"),
                        ((k.transpose(1, 2).contiguous().transpose(1, 2), v, slots, ck, cv, sc, 4), "side by side"),
                        ((k.float(), v, slots, ck, cv, sc, 4), "bf16 or fp16")):
        with pytest.raises(any4.Any4Error, match=words):
            any4.any4_kv_write(*args[:6], bits=args[6])
    with pytest.raises(any4.Any4Error, match="16-byte aligned"):                 # strides that are no multiple of 8
        odd = torch.zeros(6, 2 * 128 + 4, dtype=torch.bfloat16, device="cuda")[:, :256].view(6, 2, 128)
        any4.any4_kv_write(odd, odd, slots, ck, cv, sc, bits=4)
    with pytest.raises(any4.Any4Error, match="out"):
        any4.any4_kv_read(ck, cv, slots, sc, bits=4, out=(k[:5].contiguous(), v[:5].contiguous()))
