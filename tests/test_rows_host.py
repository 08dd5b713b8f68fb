"""The entry points for rotated rows, chunks and windows without a GPU: refusals of the C ABI (before anything touches the device) and of the
binding, and that native calls follow their tensors' device."""
import ctypes
import os
import re

import pytest
import torch

import paper_2507_04610_amd as any4
from paper_2507_04610_amd import binding
from test_attention_host import BAD_CACHES, cache, lib  # noqa: F401
from test_calls_on_another_device import calls, there  # noqa: F401

A = 0x1000                          # a 16-byte aligned address that is never read: validation fails first
NULL, SHAPE, BITS, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
NAN, INF = float("nan"), float("inf")
SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_04610_amd", "csrc", "any4_torch_rows.cpp")


def rotation(**change):
    r = dict(positions=A, axis_stride=8, freqs=A, axis_of=None, q_norm=A, k_norm=A, axes=1, rotary_dim=128, interleaved=0, eps=1e-6)
    r.update(change)
    return ctypes.byref(binding._Rotation(*(r[name] for name, _ in binding._Rotation._fields_)))


BAD_ROTATIONS = [(dict(positions=None), NULL), (dict(freqs=None), NULL), (dict(axes=0), SHAPE), (dict(axes=5), SHAPE), (dict(axis_stride=-1), SHAPE),
                 (dict(rotary_dim=0), SHAPE), (dict(rotary_dim=12), SHAPE), (dict(rotary_dim=136), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=NAN), SHAPE),
                 (dict(eps=INF), SHAPE), (dict(positions=A + 4), ALIGN), (dict(freqs=A + 4), ALIGN), (dict(q_norm=A + 2), ALIGN), (dict(k_norm=A + 8), ALIGN)]


def rope(lib, q=A, qt=512, qh=128, k=A, kt=256, kh=128, n=1, heads=4, kv_heads=2, dim=128, turn=None, qo=A, qot=512, qoh=128, ko=A, kot=256, koh=128):
    return lib.any4_rope(q, qt, qh, k, kt, kh, n, heads, kv_heads, dim, 0, turn or rotation(), qo, qot, qoh, ko, kot, koh, None)


def write(lib, q=A, qt=512, qh=128, k=A, kt=256, kh=128, v=A, vt=256, vh=128, n=1, heads=4, turn=None, slots=A, c=None, qo=A, qot=512, qoh=128, ko=None, kot=0, koh=0):
    return lib.any4_rope_kv_write(q, qt, qh, k, kt, kh, v, vt, vh, n, heads, turn or rotation(), slots, c or cache(), qo, qot, qoh, ko, kot, koh, None)


@pytest.mark.parametrize("change,code", BAD_ROTATIONS)
def test_bad_rotations_are_refused(lib, change, code):  # noqa: F811
    assert rope(lib, turn=rotation(**change)) == code and write(lib, turn=rotation(**change)) == code


def test_rope_refuses(lib):  # noqa: F811
    assert rope(lib, q=None) == rope(lib, k=None) == rope(lib, qo=None) == rope(lib, ko=None) == NULL
    assert rope(lib, n=-1) == rope(lib, n=1 << 31) == rope(lib, heads=0) == rope(lib, heads=65536) == rope(lib, kv_heads=0) == rope(lib, kv_heads=4096) == SHAPE
    assert rope(lib, dim=96) == rope(lib, qt=-8) == rope(lib, kh=-8) == rope(lib, qot=-8) == rope(lib, koh=-8) == SHAPE
    assert rope(lib, dim=64) == SHAPE                                          # (128 values to turn in heads of 64)
    assert rope(lib, q=A + 8) == rope(lib, ko=A + 2) == rope(lib, qt=516) == rope(lib, kh=4) == rope(lib, qoh=12) == ALIGN
    assert rope(lib, n=0) == 0 and rope(lib, n=0, q=None) == 0


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_bad_caches_are_refused(lib, change, code):  # noqa: F811
    assert write(lib, c=cache(**change)) == code
    assert lib.any4_attn_decode_window(A, 512, 128, cache(**change), A, 1, 1, A, 1, 4, 5, 0, 0.1, A, None, 0, None) == code


def test_rope_kv_write_refuses(lib):  # noqa: F811
    assert write(lib, q=None) == write(lib, k=None) == write(lib, v=None) == write(lib, slots=None) == write(lib, qo=None) == NULL
    assert write(lib, n=-1) == write(lib, n=1 << 31) == write(lib, heads=0) == write(lib, vt=-8) == write(lib, ko=A, kot=-8) == SHAPE
    assert write(lib, v=A + 8) == write(lib, slots=A + 4) == write(lib, vh=4) == write(lib, ko=A + 4) == write(lib, ko=A, koh=4) == ALIGN
    assert write(lib, n=0) == 0


def test_windows_are_refused(lib):  # noqa: F811
    def decode(window=5, sinks=0, n=1, scale=0.1):
        return lib.any4_attn_decode_window(A, 512, 128, cache(), A, 4, 4, A, n, 4, window, sinks, scale, A, None, 0, None)
    assert decode(window=0) == decode(window=-1) == decode(sinks=-1) == decode(scale=0.0) == decode(n=-1) == SHAPE
    assert decode(n=0) == 0


def chunk(lib, q=A, qt=512, qh=128, c=None, table=A, stride=4, width=4, starts=A, lengths=A, tokens=5, n=1, heads=4, window=0, sinks=0, scale=0.1, out=A, ws=None, size=0):  # noqa: F811
    return lib.any4_attn_chunk(q, qt, qh, c or cache(), table, stride, width, starts, lengths, tokens, n, heads, window, sinks, scale, out, ws, size, None)


def test_chunk_refuses(lib):  # noqa: F811
    assert chunk(lib, q=None) == chunk(lib, table=None) == chunk(lib, starts=None) == chunk(lib, lengths=None) == chunk(lib, out=None) == NULL
    assert chunk(lib, n=-1) == chunk(lib, tokens=-1) == chunk(lib, tokens=1 << 31) == chunk(lib, heads=3) == chunk(lib, heads=0) == chunk(lib, heads=65538) == SHAPE
    assert chunk(lib, window=-1) == chunk(lib, sinks=-1) == chunk(lib, width=0) == chunk(lib, width=1 << 28) == chunk(lib, stride=-1) == chunk(lib, qt=-8) == SHAPE
    assert chunk(lib, scale=0.0) == chunk(lib, scale=NAN) == chunk(lib, scale=INF) == chunk(lib, scale=-1.0) == SHAPE
    assert chunk(lib, tokens=1 << 30, heads=8) == SHAPE                                    # 2^32 rows of a KV head
    assert chunk(lib, tokens=1 << 29, heads=4 * 512, c=cache(kv_heads=1024)) == SHAPE      # 2^33 blocks
    assert chunk(lib, q=A + 8) == chunk(lib, table=A + 2) == chunk(lib, starts=A + 1) == chunk(lib, lengths=A + 2) == chunk(lib, out=A + 8) == chunk(lib, qt=516) == ALIGN
    assert chunk(lib, n=0) == chunk(lib, tokens=0) == 0 and chunk(lib, n=0, q=None) == 0
    need = lib.any4_attn_chunk_workspace_bytes(1, 5, 4, 2, 128, 64 * 16)
    assert need > 0 and chunk(lib, width=64) == WORKSPACE == chunk(lib, width=64, ws=A, size=need - 1) and chunk(lib, width=64, ws=A + 8, size=need) == ALIGN


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_chunk_refuses_bad_caches(lib, change, code):  # noqa: F811
    assert chunk(lib, c=cache(**change)) == code


def test_chunk_workspace(lib):  # noqa: F811
    def need(requests=3, tokens=40, heads=32, kv_heads=8, dim=128, longest=4096):
        return lib.any4_attn_chunk_workspace_bytes(requests, tokens, heads, kv_heads, dim, longest)
    assert need(longest=768) == 0 < need(longest=769)                                       # twelve tiles of keys are not cut
    assert need(requests=0) == need(tokens=0) == need(heads=30) == need(dim=96) == need(longest=0) == need(longest=1 << 31) == need(tokens=1 << 30) == 0
    # room for the pieces that a call can have, however it grows
    assert need(longest=1 << 20) <= need(tokens=1 << 20, longest=1 << 20) == need(tokens=1 << 22, longest=1 << 22) < 160 << 20
    assert need(dim=64) < need()
    assert 0 < need(requests=65, longest=64) < need(requests=1000, longest=64) < 1 << 15       # (where the requests' blocks end)


def test_prompt_window_refuses(lib):  # noqa: F811
    def prompt(q=A, qt=512, qh=128, k=A, kt=256, kh=128, v=A, vt=256, vh=128, nq=5, nk=7, qs=A, ks=A, n=1, heads=4, kv=2, dim=128, window=4, sinks=0, scale=0.1, out=A):
        return lib.any4_attn_prompt_window(q, qt, qh, k, kt, kh, v, vt, vh, nq, nk, qs, ks, n, heads, kv, dim, 0, window, sinks, scale, out, None)
    assert prompt(q=None) == prompt(k=None) == prompt(v=None) == prompt(qs=None) == prompt(ks=None) == prompt(out=None) == NULL
    assert prompt(window=0) == prompt(window=-1) == prompt(sinks=-1) == prompt(n=-1) == prompt(nq=-1) == prompt(nk=1 << 31) == prompt(heads=3) == prompt(dim=96) == SHAPE
    assert prompt(scale=0.0) == prompt(kt=1 << 23) == prompt(vt=1 << 23) == prompt(vh=-8) == prompt(nq=1 << 30, heads=8) == SHAPE
    assert prompt(q=A + 8) == prompt(k=A + 2) == prompt(qs=A + 2) == prompt(vh=4) == prompt(out=A + 4) == ALIGN
    assert prompt(n=0) == prompt(nq=0) == 0


def test_the_binding_names_the_mistake():
    q, k, where, freqs = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64), torch.ones(64, dtype=torch.float64)
    with pytest.raises(any4.Any4Error, match="device memory"):
        any4.any4_rope(q, k, where, freqs)
    with pytest.raises(any4.Any4Error, match="pair of tensors"):
        any4.any4_rope(q, k, where, freqs, out=q)
    with pytest.raises(any4.Any4Error, match="3 dimensions"):
        any4.any4_rope(q[0], k, where, freqs)
    with pytest.raises(any4.Any4Error, match="sinks"):
        any4.any4_attn_decode(q, None, None, None, None, sinks=3)
    for bad in (0, -1, 2.0, True, "5"):
        with pytest.raises(any4.Any4Error, match="window"):
            any4.any4_attn_decode(q, None, None, None, None, window=bad)
    with pytest.raises(any4.Any4Error, match="sinks"):
        any4.any4_attn_decode(q, None, None, None, None, window=4, sinks=-1)


def turned(**change):
    a = dict(q=there(3, 4, 128), k=there(3, 2, 128), positions=there(3, dtype=torch.int64), freqs=there(64, dtype=torch.float64))
    a.update(change)
    return any4.any4_rope(**a)


BAD = [("positions", dict(positions=there(4, dtype=torch.int64))), ("positions", dict(positions=there(3, dtype=torch.int32))), ("positions", dict(positions=there(3, 2, dtype=torch.int64))),
       ("1 to 4", dict(positions=there(5, 3, dtype=torch.int64))), ("freqs", dict(freqs=there(64, dtype=torch.float32))), ("freqs", dict(freqs=there(3, dtype=torch.float64))),
       ("freqs", dict(freqs=there(68, dtype=torch.float64))), ("freqs", dict(freqs=there(0, dtype=torch.float64))), ("q_norm", dict(q_norm=there(64))),
       ("k_norm", dict(k_norm=there(128, dtype=torch.float16))), ("axis_of", dict(axis_of=there(32, dtype=torch.uint8))), ("k must have", dict(k=there(4, 2, 128))),
       ("k must have", dict(k=there(3, 2, 128, dtype=torch.float16))), ("bf16 or fp16", dict(q=there(3, 4, 128, dtype=torch.float32))),
       ("overlap", dict(out=(there(1, 4, 128).expand(3, 4, 128), there(3, 2, 128)))), ("overlap", dict(out=(there(3, 4, 128), there(3, 1, 128).expand(3, 2, 128)))),
       ("out", dict(out=(there(3, 4, 64), there(3, 2, 128))))]


@pytest.mark.parametrize("words,change", BAD)
def test_bad_tensors_are_refused(calls, words, change):  # noqa: F811
    with pytest.raises(any4.Any4Error, match=words):
        turned(**change)
    assert not calls


def test_calls_run_where_the_tensors_lie(calls):  # noqa: F811
    turned()
    turned(out=(there(4, 3, 128).transpose(0, 1), there(3, 5, 136)[:, 1:3, :128]))
    ck, cv, table, i32 = there(4, 2, 16, 128), there(4, 2, 16, 128), there(3, 2, dtype=torch.int32), there(3, dtype=torch.int32)
    q, k, i64 = there(3, 4, 128), there(3, 2, 128), there(3, dtype=torch.int64)
    any4.any4_rope_kv_write(q, k, k, there(3, 3, dtype=torch.int64), there(64, dtype=torch.float64), i64, ck, cv, axis_of=there(64, dtype=torch.uint8))
    any4.any4_attn_decode(q, ck, cv, table, i32, window=7, sinks=2)
    any4.any4_attn_chunk(q, ck, cv, table, there(4, dtype=torch.int32), i32)
    any4.any4_attn_prompt(q, k, k, i32, window=7)
    names = [name for name, _, _ in calls]
    assert names == ["any4_rope", "any4_rope", "any4_rope_kv_write", "any4_attn_decode_workspace_bytes", "any4_attn_decode_window",
                     "any4_attn_chunk_workspace_bytes", "any4_attn_chunk", "any4_attn_prompt_window"]
    assert all(device == 1 and stream in (101, None) for _, device, stream in calls) and torch.cuda.current_device() == 0


def test_native_calls_switch_to_the_tensors_device_and_let_go_of_the_lock():
    with open(SOURCE) as f:
        text = f.read()
    bodies = re.findall(r"(?ms)^PyObject\* (\w+)\(PyObject\*, PyObject\* const\* a, Py_ssize_t n\) \{(.*?)^\}", text)
    assert {"rope", "rope_kv_write", "attn_decode_window", "attn_chunk", "attn_prompt_window"} == {name for name, _ in bodies}
    for name, body in bodies:
        switch = body.index("stream_on(")
        for later in ("at::empty(", "_workspace_bytes("):
            assert later not in body or body.index(later) > switch, (name, later)
        unlocked = body[body.index("Py_BEGIN_ALLOW_THREADS"):body.index("Py_END_ALLOW_THREADS")]
        assert re.findall(r"= any4_\w+\(", unlocked) == re.findall(r"= any4_(?!\w*_bytes)\w+\(", body), name


def test_host_tensors_are_left_to_the_checked_calls():
    any4.load_library()
    n = binding._native_calls
    q, k, i64, f = torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64), torch.ones(64, dtype=torch.float64)
    ck = torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16)
    assert n.rope(q, k, i64, f, None, None, 1e-6, False, None, None, None) is None
    assert n.rope_kv_write(q, k, k, i64, f, i64, ck, ck, None, 16, None, None, 1e-6, False, None, None, None) is None
    assert n.attn_chunk(q, ck, ck, i64[:, None].int(), torch.zeros(4).int(), i64.int(), None, 16, 0, 0, None, None, None) is None
    assert n.attn_prompt_window(q, k, k, i64.int(), None, 4, 0, None, None) is None
    assert n.attn_decode_window(q, ck, ck, i64[:, None].int(), i64.int(), None, 16, None, None, None, 5, 0) is None


BAD_CHUNKS = [("3 dimensions", dict(q=there(3, 128))), ("multiple", dict(q=there(3, 3, 128))), ("lengths", dict(lengths=there(2, dtype=torch.int64))),
              ("lengths", dict(lengths=there(2, 1, dtype=torch.int32))), ("q_starts", dict(q_starts=there(2, dtype=torch.int32))), ("q_starts", dict(q_starts=there(3, dtype=torch.int64))),
              ("page_table", dict(page_table=there(2, 2))), ("page_table", dict(page_table=there(3, 2, dtype=torch.int32))), ("out", dict(out=there(3, 4, 64))),
              ("cache_v", dict(cache_v=there(4, 2, 16, 64))), ("bits", dict(bits=5)), ("scales", dict(bits=8, cache_k=there(4, 2, 16, 128, dtype=torch.uint8), cache_v=there(4, 2, 16, 128, dtype=torch.uint8),
                                                                                                     scales=there(4, 2, 16, 2))),
              ("workspace", dict(workspace=torch.zeros(8))), ("sinks", dict(sinks=4)), ("window", dict(window=0))]


@pytest.mark.parametrize("words,change", BAD_CHUNKS)
def test_bad_chunks_are_refused(calls, words, change):  # noqa: F811
    a = dict(q=there(3, 4, 128), cache_k=there(4, 2, 16, 128), cache_v=there(4, 2, 16, 128), page_table=there(2, 2, dtype=torch.int32), q_starts=there(3, dtype=torch.int32),
             lengths=there(2, dtype=torch.int32))
    a.update(change)
    with pytest.raises(any4.Any4Error, match=words):
        any4.any4_attn_chunk(**a)
    assert not [name for name, _, _ in calls if "bytes" not in name]
