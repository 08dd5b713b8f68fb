"""The entry points of the key-value cache and of attention without a GPU: refusals of the C ABI (before anything touches the
device) and of the binding, workspace sizes, the layout's reference."""
import ctypes
import os

import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2507_04610_amd as any4
from paper_2507_04610_amd import binding

A = 0x1000                          # a 16-byte aligned address that is never read: validation fails first
NULL, SHAPE, BITS, ALIGN, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_04610_amd import build
        build.build_library(verbose=False)
    return binding.load_library()


def cache(**change):
    c = dict(k=A, v=A, scales=A, pages=4, page_size=16, kv_heads=2, head_dim=128, bits=8, f16=0)
    c.update(change)
    return ctypes.byref(binding._KvCache(*(c[name] for name, _ in binding._KvCache._fields_)))


BAD_CACHES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(scales=None), NULL), (dict(bits=3), BITS), (dict(bits=0), BITS),
              (dict(pages=0), SHAPE), (dict(pages=1 << 31), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE),
              (dict(page_size=2048), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=4096), SHAPE), (dict(head_dim=96), SHAPE),
              (dict(k=A + 8), ALIGN), (dict(v=A + 4), ALIGN), (dict(scales=A + 2), ALIGN)]


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_bad_caches_are_refused_by_every_entry_point(lib, change, code):
    c = cache(**change)
    assert lib.any4_kv_write(A, 256, 128, A, 256, 128, 1, A, c, None) == code
    assert lib.any4_kv_read(c, A, 1, A, A, None) == code
    assert lib.any4_attn_decode(A, 512, 128, c, A, 1, 1, A, 1, 4, 0.1, A, None, 0, None) == code


def test_write_and_read_refuse(lib):
    def write(k=A, kt=256, kh=128, v=A, vt=256, vh=128, n=1, slots=A):
        return lib.any4_kv_write(k, kt, kh, v, vt, vh, n, slots, cache(), None)
    assert write(k=None) == write(v=None) == write(slots=None) == NULL
    assert write(n=-1) == write(n=1 << 31) == write(kt=-256) == write(vh=-8) == SHAPE
    assert write(k=A + 2) == write(v=A + 8) == write(slots=A + 4) == write(kt=132) == write(vh=4) == ALIGN
    assert write(n=0) == 0 and write(n=0, k=None) == 0
    assert lib.any4_kv_read(cache(), None, 1, A, A, None) == lib.any4_kv_read(cache(), A, 1, None, A, None) == NULL
    assert lib.any4_kv_read(cache(), A, 1, A, A + 8, None) == ALIGN and lib.any4_kv_read(cache(), A, -1, A, A, None) == SHAPE
    assert lib.any4_kv_read(cache(), None, 0, None, None, None) == 0
    assert lib.any4_kv_write(A, 256, 128, A, 256, 128, 0, A, None, None) == NULL


def test_decode_refuses(lib):
    def decode(q=A, qt=512, qh=128, c=None, table=A, stride=4, width=4, lengths=A, n=1, heads=4, scale=0.1, out=A, ws=None, size=0):
        return lib.any4_attn_decode(q, qt, qh, c or cache(), table, stride, width, lengths, n, heads, scale, out, ws, size, None)
    assert decode(q=None) == decode(table=None) == decode(lengths=None) == decode(out=None) == NULL
    for bad in (dict(n=-1), dict(n=65536), dict(heads=3), dict(heads=0), dict(heads=65536), dict(width=0), dict(width=1 << 40), dict(stride=-1), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(qt=-8)):
        assert decode(**bad) == SHAPE, bad
    for bad in (dict(q=A + 8), dict(out=A + 2), dict(table=A + 2), dict(lengths=A + 1), dict(qt=516), dict(qh=4), dict(ws=A + 4)):
        assert decode(**bad) == ALIGN, bad
    assert decode(n=0) == 0
    need = lib.any4_attn_decode_workspace_bytes(1, 4, 2, 128, 65536)
    assert need > 0 and need % 4 == 0
    assert decode(width=4096) == WORKSPACE and decode(width=4096, ws=A, size=need - 1) == WORKSPACE


def test_workspace_bytes(lib):
    f = lib.any4_attn_decode_workspace_bytes
    assert f(0, 4, 2, 128, 64) == f(1, 3, 2, 128, 64) == f(1, 4, 2, 96, 64) == f(1, 4, 2, 128, 0) == f(65536, 4, 2, 128, 64) == 0
    assert f(1, 4, 2, 128, 16) == 0                                     # one piece: nothing to join
    assert f(1, 32, 8, 128, 131072) < 64 << 20
    assert any4.any4_attn_decode_workspace_bytes(1, 4, 2, 128, 65536) == f(1, 4, 2, 128, 65536)


def test_prompt_refuses(lib):
    def prompt(q=A, qt=512, qh=128, k=A, kt=256, kh=128, v=A, vt=256, vh=128, nq=5, nk=5, qs=A, ks=A, n=1, heads=4, kv=2, dim=128, scale=0.1, out=A):
        return lib.any4_attn_prompt(q, qt, qh, k, kt, kh, v, vt, vh, nq, nk, qs, ks, n, heads, kv, dim, 0, 1, scale, out, None)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(qs=None), dict(ks=None), dict(out=None)):
        assert prompt(**bad) == NULL, bad
    for bad in (dict(nq=-1), dict(nk=1 << 31), dict(n=-1), dict(heads=3), dict(kv=0), dict(dim=80), dict(scale=0.0), dict(scale=float("nan")),
                dict(kt=1 << 23), dict(vt=1 << 23), dict(qh=-8)):
        assert prompt(**bad) == SHAPE, bad
    for bad in (dict(q=A + 8), dict(v=A + 2), dict(qs=A + 2), dict(out=A + 4), dict(qt=1), dict(kh=4), dict(vt=20)):
        assert prompt(**bad) == ALIGN, bad
    assert prompt(nq=0x7FFFFFFF - 2047, nk=0x7FFFFFFF - 2047, heads=256) == SHAPE          # more blocks than a launch has
    assert prompt(n=0) == prompt(nq=0) == prompt(nq=0, q=None) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    ck, cv, scales = any4.any4_kv_cache(2, 2, 128, 16, bits=8, device="cpu")
    assert ck.shape == (2, 2, 16, 128) and ck.dtype == torch.uint8 and scales.shape == (2, 2, 16, 4)
    assert any4.any4_kv_cache(2, 2, 128, 16, bits=4, device="cpu")[0].shape == (2, 2, 16, 64)
    assert any4.any4_kv_cache(2, 2, 64, 16, dtype=torch.float16, device="cpu")[2] is None
    slots = torch.arange(3)
    with pytest.raises(any4.Any4Error, match="bits"):
        any4.any4_kv_cache(2, 2, 128, 16, bits=3)
    with pytest.raises(any4.Any4Error, match="device memory"):
        any4.any4_kv_write(k, k, slots, ck, cv, scales, bits=8)
    with pytest.raises(any4.Any4Error, match="device memory"):
        any4.any4_kv_read(ck, cv, slots, scales, bits=8)
    with pytest.raises(any4.Any4Error, match="device memory"):
        any4.any4_attn_decode(k, ck, cv, torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), scales, bits=8)
    with pytest.raises(any4.Any4Error, match="device memory"):
        any4.any4_attn_prompt(k, k, k, torch.tensor([0, 3], dtype=torch.int32))
    with pytest.raises(any4.Any4Error, match="3 dimensions"):
        any4.any4_attn_prompt(k[0], k, k, torch.tensor([0, 3], dtype=torch.int32))
    with pytest.raises(any4.Any4Error, match="bf16 or fp16"):
        any4.any4_attn_prompt(k.float(), k, k, torch.tensor([0, 3], dtype=torch.int32))


def test_reference_encoding_by_hand():
    x = np.array([[0.0, 1.0, 2.0, 15.0], [-8.0, 7.0, 0.5, 1.5], [3.0, 3.0, 3.0, 3.0], [np.inf, 0.0, 0.0, 0.0]], np.float32)
    codes, scale, offset = ref.encode(x, 4)
    assert codes[0].tolist() == [0, 1, 2, 15] and scale[0] == 1 and offset[0] == 0
    assert codes[1].tolist() == [0, 15, 8, 10] and offset[1] == -8      # 8.5 and 9.5: ties to even
    assert codes[2].tolist() == [0, 0, 0, 0] and scale[2] == 1 and offset[2] == 3
    assert np.isnan(scale[3, 0]) and np.isnan(offset[3, 0]) and not codes[3].any()
    assert np.array_equal(ref.unpack(ref.pack(codes, 4), 4), codes)
