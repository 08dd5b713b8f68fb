"""Calls whose tensors lie on another device than the current one run on theirs, on its stream, with workspaces of its size: the binding
with tensors that claim to lie on a second device and a library that notes what is current, the native calls by their text."""
import contextlib
import os
import re
import types

import pytest
import torch

import paper_2507_04610_amd as any4
from paper_2507_04610_amd import binding

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_04610_amd", "csrc", "any4_torch.cpp")


class There(torch.Tensor):
    """host memory that says it lies on cuda:1"""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 1))


def there(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(There)


@pytest.fixture()
def calls(monkeypatch):
    """[(entry point, current device, stream)] of the calls that reach the library"""
    now, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d.index
        yield
        now[0] = before

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                seen.append((name, now[0], None if "_bytes" in name else args[-1]))
                return 4096 if "_bytes" in name else 0
            return entry
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=100 + now[0], device_index=now[0]))
    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "_native_gemm", binding._no_native_gemm)
    monkeypatch.setattr(binding, "_native_calls", binding._NoNativeCalls)
    # (what the binding allocates lies there as well)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw).as_subclass(There))
    return seen


def cache_calls():
    k, i32, i64 = there(3, 2, 128), there(3, dtype=torch.int32), there(3, dtype=torch.int64)
    ck, cv, table = there(4, 2, 16, 128), there(4, 2, 16, 128), there(3, 2, dtype=torch.int32)
    any4.any4_kv_write(k, k, i64, ck, cv)
    any4.any4_kv_read(ck, cv, i64)
    any4.any4_attn_decode(k, ck, cv, table, i32)
    any4.any4_attn_prompt(k, k, k, i32)


def linear_calls():
    codes, lut, s = there(64, 32, dtype=torch.int32), there(64, 16), there(64, 2)
    any4.any4_gemm(there(2, 256), codes, lut, s, s, 4)
    any4.any4_gemm_noalloc(there(2, 256), codes, lut, s, s, 4)
    any4.any4_pack(there(64, 256, dtype=torch.uint8), 4)
    any4.any4_dequant(codes, lut, s, s, 256, 4)
    any4.any4_repack(codes, 4)
    any4.any4_quantize(there(64, 256, dtype=torch.float32), None, there(64, 16, dtype=torch.float32), 4)


@pytest.mark.parametrize("some,names", [
    (cache_calls, ["any4_kv_write", "any4_kv_read", "any4_attn_decode_workspace_bytes", "any4_attn_decode", "any4_attn_prompt"]),
    (linear_calls, ["any4_gemm_workspace_bytes", "any4_gemm", "any4_gemm_noalloc", "any4_pack", "any4_dequant", "any4_quantize"])])
def test_calls_run_where_the_tensors_lie(calls, some, names):
    some()
    assert set(names) <= {name for name, _, _ in calls}
    for name, device, stream in calls:
        if name != "any4_repack_bytes":                         # (the same for every device)
            assert device == 1 and stream in (101, None), (name, device, stream)
    assert torch.cuda.current_device() == 0


def test_native_calls_switch_to_the_tensors_device():
    with open(SOURCE) as f:
        text = f.read()
    on = re.search(r"(?ms)^void\* stream_on\(.*?^\}", text).group(0)
    assert re.search(r"if \(.*device_index\(\) != device\.index\(\)\).*reset_device\(device\);.*getCurrentHIPStream\(\)", on, re.S)
    bodies = re.findall(r"(?ms)^PyObject\* (\w+)\(PyObject\*, PyObject\* const\* a, Py_ssize_t n\) \{(.*?)^\}", text)
    assert {name for name, _ in bodies} == {"gemm", "kv_write", "kv_read", "attn_decode", "attn_prompt"}
    for name, body in bodies:
        switch = body.index("stream_on(")
        assert "getCurrentHIPStream" not in body
        for later in ("at::empty(", "_workspace_bytes("):
            assert later not in body or body.index(later) > switch, (name, later)
        # ... and let other threads run while they launch
        unlocked = body[body.index("Py_BEGIN_ALLOW_THREADS"):body.index("Py_END_ALLOW_THREADS")]
        assert re.findall(r"= any4_\w+\(", unlocked) == re.findall(r"= any4_(?!\w*_bytes)\w+\(", body), name
