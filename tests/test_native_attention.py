"""The native calls of the cache and of attention (csrc/any4_torch.cpp) against the checked Python calls they stand in for: the
same bits, and a plain "no" to whatever the Python call refuses; without the extension every entry point is still there."""
import pytest
import torch

import paper_2507_04610_amd as any4
from paper_2507_04610_amd import binding


def problem(bits, dtype, device="cuda"):
    g = torch.Generator().manual_seed(bits)
    row = torch.randn(70, 8 * 64, generator=g).to(dtype).to(device)
    q, k, v = row[:, :256].view(70, 4, 64), row[:, 256:384].view(70, 2, 64), row[:, 384:].view(70, 2, 64)
    cache = any4.any4_kv_cache(6, 2, 64, 16, bits, dtype, device)
    slots = torch.arange(70, device=device) + 9
    table = torch.arange(6, dtype=torch.int32, device=device).expand(3, 6).contiguous()
    return q, k, v, cache, slots, table, torch.tensor([79, 5, 0], dtype=torch.int32, device=device), torch.tensor([0, 30, 70], dtype=torch.int32, device=device)


def everything(bits, dtype):
    q, k, v, (ck, cv, sc), slots, table, lengths, starts = problem(bits, dtype)
    any4.any4_kv_write(k, v, slots, ck, cv, sc, bits=bits)
    out = torch.empty(3, 4, 64, dtype=dtype, device="cuda")
    pair = tuple(torch.empty(70, 2, 64, dtype=dtype, device="cuda") for _ in range(2))
    return [ck, cv, *([sc] if bits != 16 else []), *any4.any4_kv_read(ck, cv, slots, sc, bits=bits, dtype=dtype),
            *any4.any4_kv_read(ck, cv, slots, sc, bits=bits, dtype=dtype, out=pair),
            any4.any4_attn_decode(q[:3], ck, cv, table, lengths, sc, bits=bits), any4.any4_attn_decode(q[:3], ck, cv, table, lengths, sc, bits=bits, out=out),
            any4.any4_attn_decode(q[:3], ck, cv, table, lengths, sc, bits=bits, softmax_scale=0.5),
            any4.any4_attn_prompt(q, k, v, starts), any4.any4_attn_prompt(q, k, v, starts, starts, causal=False, softmax_scale=0.25, out=torch.empty_like(q.contiguous()))]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
def test_native_calls_give_the_bits_of_the_checked_calls(bits, dtype, monkeypatch):
    native = everything(bits, dtype)
    monkeypatch.setattr(binding, "_native_calls", binding._NoNativeCalls)
    for a, b in zip(native, everything(bits, dtype)):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
def test_valid_calls_are_native():
    q, k, v, (ck, cv, sc), slots, table, lengths, starts = problem(8, torch.bfloat16)
    any4.load_library()
    n = binding._native_calls
    out = torch.empty(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert n.kv_write(k, v, slots, ck, cv, sc, 8) is True
    assert n.kv_read(ck, cv, slots, sc, 8, False, None, None)[0].shape == (70, 2, 64)
    assert n.attn_decode(q[:3], ck, cv, table, lengths, sc, 8, None, out, None) is out
    assert n.attn_prompt(q, k, v, starts, None, True, None, None).shape == (70, 4, 64)
    # ... and what is not valid is nobody's call
    assert n.kv_write(k, v, slots[:5], ck, cv, sc, 8) is None
    assert n.kv_write(k, v, slots, ck, cv, None, 8) is None
    assert n.kv_read(ck, cv, slots, sc, 4, False, None, None)[0].shape == (70, 2, 128)       # (the same bytes are twice as many codes of 4 bits)
    assert n.kv_read(ck, cv, slots.int(), sc, 8, False, None, None) is None
    assert n.kv_read(ck, cv, slots, sc, 8, False, out, None) is None
    assert n.attn_decode(q[:3], ck, cv, table, lengths, sc, 8, 0.0, None, None) is None
    assert n.attn_decode(q[:2], ck, cv, table, lengths, sc, 8, None, None, None) is None
    assert n.attn_decode(q[:3].half(), ck, cv, table, lengths, sc, 16, None, None, None) is None
    assert n.attn_prompt(q, k[:5], v[:5], starts, None, True, None, None) is None
    assert n.attn_prompt(q, k, v, starts.long(), None, True, None, None) is None


def test_host_tensors_are_left_to_the_checked_calls():
    q, k, v, (ck, cv, sc), slots, table, lengths, starts = problem(8, torch.bfloat16, "cpu")
    any4.load_library()
    n = binding._native_calls
    assert n.kv_write(k, v, slots, ck, cv, sc, 8) is None and n.kv_read(ck, cv, slots, sc, 8, False, None, None) is None
    assert n.attn_decode(q[:3], ck, cv, table, lengths, sc, 8, None, None, None) is None
    assert n.attn_prompt(q, k, v, starts, None, True, None, None) is None


def test_stand_ins_say_no():
    assert binding._NoNativeCalls.kv_write(1, 2) is None and binding._NoNativeCalls.attn_prompt() is None
