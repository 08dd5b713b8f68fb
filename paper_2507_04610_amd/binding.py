"""Thin Python binding of libany4's C ABI (include/any4.h).

Argument marshalling only: every function takes torch tensors that already live in device
memory, checks dtype / shape / contiguity (every array the kernels index is compared with the
shape (N, K, bits, group) implies), and passes raw pointers plus the current HIP stream of
the tensors' device to the library.  No arithmetic of the method happens here, and there is no fallback: if the
shared library is missing or a call is made with host tensors, this module raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libany4.so")
GROUP = 128

EXPORTS = ("any4_pack", "any4_dequant", "any4_gemm", "any4_gemm_workspace_bytes", "any4_repack", "any4_repack_bytes", "any4_gemm_repacked", "any4_dequant_grouped", "any4_gemm_grouped", "any4_dequant_f16", "any4_gemm_f16",
           "any4_quantize", "any4_quantize_with_gap", "any4_quantize_max_k", "any4_gemm_noalloc", "any4_dequant_single_table", "any4_gemm_single_table",
           "any4_kv_write", "any4_kv_read", "any4_attn_decode", "any4_attn_decode_workspace_bytes", "any4_attn_prompt", "any4_strerror", "any4_version")


class Any4Error(RuntimeError):
    pass


class _KvCache(ctypes.Structure):
    """any4_kv_cache of include/any4.h"""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("pages", ctypes.c_int64),
                ("page_size", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("bits", ctypes.c_int),
                ("f16", ctypes.c_int)]


_lib = None
_native_gemm = None          # the native call (_any4_torch.gemm) once the library is loaded
_native_calls = None         # the native calls of the cache and of attention (_any4_torch), likewise


def load_library() -> ctypes.CDLL:
    """Load libany4.so from the package directory (build it with
    `python -m paper_2507_04610_amd.build`); raises if it is not there."""
    global _lib, _native_gemm, _native_calls
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise Any4Error(f"{LIB_PATH} is missing: run `python -m paper_2507_04610_amd.build` first")
    lib = ctypes.CDLL(LIB_PATH)
    i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.any4_pack.restype = ci
    lib.any4_pack.argtypes = [vp, i64, i64, ci, vp, vp]
    lib.any4_dequant.restype = ci
    lib.any4_dequant.argtypes = [vp, vp, vp, vp, i64, i64, ci, vp, vp]
    lib.any4_gemm.restype = ci
    lib.any4_gemm.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, vp, vp, ctypes.c_size_t, vp]
    lib.any4_gemm_workspace_bytes.restype = ctypes.c_size_t
    lib.any4_gemm_workspace_bytes.argtypes = [i64, i64, i64, ci]
    lib.any4_dequant_grouped.restype = ci
    lib.any4_dequant_grouped.argtypes = [vp, vp, vp, vp, i64, i64, ci, ci, vp, vp]
    lib.any4_dequant_f16.restype = ci
    lib.any4_dequant_f16.argtypes = [vp, vp, vp, vp, i64, i64, ci, vp, vp]
    lib.any4_gemm_f16.restype = ci
    lib.any4_gemm_f16.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, vp, vp, ctypes.c_size_t, vp]
    lib.any4_gemm_grouped.restype = ci
    lib.any4_gemm_grouped.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, ci, vp, vp, ctypes.c_size_t, vp]
    lib.any4_gemm_repacked.restype = ci
    lib.any4_gemm_repacked.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, vp, vp, ctypes.c_size_t, vp]
    lib.any4_dequant_single_table.restype = ci
    lib.any4_dequant_single_table.argtypes = [vp, vp, vp, vp, i64, i64, ci, vp, vp]
    lib.any4_gemm_single_table.restype = ci
    lib.any4_gemm_single_table.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, vp, vp, ctypes.c_size_t, vp]
    lib.any4_gemm_noalloc.restype = ci
    lib.any4_gemm_noalloc.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ci, vp, vp]
    lib.any4_repack.restype = ci
    lib.any4_repack.argtypes = [vp, i64, i64, ci, vp, vp]
    lib.any4_repack_bytes.restype = ctypes.c_size_t
    lib.any4_repack_bytes.argtypes = [i64, i64, ci]
    lib.any4_quantize.restype = ci
    lib.any4_quantize.argtypes = [vp, vp, vp, i64, i64, ci, ci, ci, vp, vp, vp, vp, vp, vp]
    lib.any4_quantize_with_gap.restype = ci
    lib.any4_quantize_with_gap.argtypes = [vp, vp, vp, i64, i64, ci, ci, ci, ctypes.c_double, vp, vp, vp, vp, vp, vp]
    lib.any4_quantize_max_k.restype = i64
    lib.any4_quantize_max_k.argtypes = []
    cache, f32 = ctypes.POINTER(_KvCache), ctypes.c_float
    lib.any4_kv_write.restype = ci
    lib.any4_kv_write.argtypes = [vp, i64, i64, vp, i64, i64, i64, vp, cache, vp]
    lib.any4_kv_read.restype = ci
    lib.any4_kv_read.argtypes = [cache, vp, i64, vp, vp, vp]
    lib.any4_attn_decode.restype = ci
    lib.any4_attn_decode.argtypes = [vp, i64, i64, cache, vp, i64, i64, vp, i64, ci, f32, vp, vp, ctypes.c_size_t, vp]
    lib.any4_attn_decode_workspace_bytes.restype = ctypes.c_size_t
    lib.any4_attn_decode_workspace_bytes.argtypes = [i64, ci, ci, ci, i64]
    lib.any4_attn_prompt.restype = ci
    lib.any4_attn_prompt.argtypes = [vp, i64, i64, vp, i64, i64, vp, i64, i64, i64, i64, vp, vp, i64, ci, ci, ci, ci, ci, f32, vp, vp]
    lib.any4_strerror.restype = ctypes.c_char_p
    lib.any4_strerror.argtypes = [ci]
    lib.any4_version.restype = ci
    lib.any4_version.argtypes = []
    problem = None
    try:
        from . import _any4_torch as native
        gemm, calls = native.gemm, native
    except ImportError as e:
        # built for another torch, or not built: the checked calls run the same kernels, only the call costs more
        gemm, calls, problem = _no_native_gemm, _NoNativeCalls, str(e)
    _native_gemm, _native_calls = gemm, calls
    _lib = lib                   # last: another thread that sees it finds the call as well
    if problem:
        warnings.warn(f"the torch extension beside {LIB_PATH} does not load ({problem}): GEMM calls go through ctypes; "
                      "`python -m paper_2507_04610_amd.build` builds it", RuntimeWarning, stacklevel=2)
    return lib


def _no_native_gemm(*args):
    """in the place of the native call where its extension does not load: never a plain valid call"""
    return None


class _NoNativeCalls:
    """the same for the cache and attention"""
    kv_write = kv_read = attn_decode = attn_prompt = staticmethod(_no_native_gemm)


def _calls():
    """the native calls (csrc/any4_torch.cpp): each gives its result, None with nothing done where a call is not a plain valid
    one (the checked call then names what is wrong), or a code from the runtime"""
    if _native_calls is None:
        load_library()
    return _native_calls


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise Any4Error(f"{what} failed: {load_library().any4_strerror(rc).decode()} ({rc})")


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise Any4Error(f"{name} must be a tensor in device memory")
    if t.dtype != dtype:
        raise Any4Error(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise Any4Error(f"{name} must be contiguous")
    return t.data_ptr()


def _shape(t: torch.Tensor, want, name: str) -> None:
    if tuple(t.shape) != tuple(want):
        raise Any4Error(f"{name} must have shape {tuple(want)}, got {tuple(t.shape)}")


def _check_quant_shapes(codes, lut, scale, offset, N, K, bits, group, repacked=False, single_table=False) -> None:
    """the kernels index these arrays from (N, K, bits, group) alone: a wrong shape would make them read
    out of bounds on the device, so it is refused here"""
    if bits not in (4, 3, 2):
        raise Any4Error(f"bits must be 4, 3 or 2, got {bits}")
    if K < 1 or K % GROUP or group < 1 or K % group:
        raise Any4Error(f"K = {K} must be a positive multiple of 128 and of the group size {group}")
    if repacked:
        need = (N + 15) // 16 * 16 * row_words(K, bits)
        if codes.numel() != need:
            raise Any4Error(f"rcodes must hold {need} words (any4_repack_bytes), got {codes.numel()}")
    else:
        _shape(codes, (N, row_words(K, bits)), "codes")
    if lut is not None and not (single_table and tuple(lut.shape) == (1, 1 << bits)):
        _shape(lut, (N, 1 << bits), "lut")
    _shape(scale, (N, K // group), "scale")
    _shape(offset, (N, K // group), "offset")


def _scratch(t, device) -> tuple[int, int]:
    """address and bytes of a caller's workspace, which the kernels write: memory of x's device, as much of it as the
    tensor has elements (an expanded tensor has fewer, a strided one has another's elements in between)"""
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise Any4Error(f"workspace must be a tensor on x's device, {device}")
    if t.numel() > 0 and sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1 != t.numel():
        raise Any4Error("workspace must be one piece of memory (contiguous)")
    return t.data_ptr(), t.numel() * t.element_size()


def _launch(entry: str, device, *args) -> None:
    """the entry point on the tensors' device, on torch's current stream of it"""
    stream = torch.cuda.current_stream()
    if stream.device_index != device.index:
        with torch.cuda.device(device):
            return _launch(entry, device, *args)
    rc = getattr(load_library(), entry)(*args, stream.cuda_stream)
    if rc != 0:
        _check(rc, entry)


def _bytes_on(device, entry: str, *args) -> int:
    """a workspace's size, which depends on the device"""
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _bytes_on(device, entry, *args)
    return int(getattr(load_library(), entry)(*args))


def row_words(K: int, bits: int) -> int:
    return K * bits // 32


def any4_version() -> int:
    return int(load_library().any4_version())


def any4_strerror(code: int) -> str:
    return load_library().any4_strerror(code).decode()


def any4_gemm_workspace_bytes(M: int, N: int, K: int, bits: int = 4) -> int:
    return int(load_library().any4_gemm_workspace_bytes(M, N, K, bits))


def any4_pack(codes_u8: torch.Tensor, bits: int = 4, out: torch.Tensor | None = None) -> torch.Tensor:
    """uint8 [N,K] codes (one per byte) -> packed words, int32 tensor [N, K*bits/32]
    (torch has no usable uint32; the bit patterns are what matters)."""
    N, K = codes_u8.shape
    src = _dev(codes_u8, torch.uint8, "codes_u8")
    if out is None:
        out = torch.empty((N, max(K * bits // 32, 0)), dtype=torch.int32, device=codes_u8.device)
    _shape(out, (N, max(K * bits // 32, 0)), "out")
    dst = _dev(out, torch.int32, "out")
    _launch("any4_pack", codes_u8.device, src, N, K, bits, dst)
    return out


def any4_dequant(codes: torch.Tensor, lut: torch.Tensor | None, scale: torch.Tensor, offset: torch.Tensor,
                 K: int, bits: int = 4, out: torch.Tensor | None = None, group: int = GROUP) -> torch.Tensor:
    """fp32 [N,K] dequantised weights (lut None with bits 4: the int4 grid, value = code - 8; lut of
    shape [1, 2^bits]: one table for the whole matrix);
    scale / offset are [N, K / group] (any4_dequant_grouped when group is not 128).
    lut / scale / offset are bf16, or all fp16 (any4_dequant_f16: groups of 128, a table)."""
    N = codes.shape[0]
    pc = _dev(codes, torch.int32, "codes")
    dt = scale.dtype if isinstance(scale, torch.Tensor) and scale.dtype == torch.float16 else torch.bfloat16
    single = lut is not None and N != 1 and tuple(lut.shape) == (1, 1 << bits)
    _check_quant_shapes(codes, lut, scale, offset, N, K, bits, group, single_table=single)
    pl = _dev(lut, dt, "lut") if lut is not None else None
    ps = _dev(scale, dt, "scale")
    po = _dev(offset, dt, "offset")
    if out is None:
        out = torch.empty((N, K), dtype=torch.float32, device=codes.device)
    _shape(out, (N, K), "out")
    pw = _dev(out, torch.float32, "out")
    if single:
        if dt == torch.float16 or group != GROUP:
            raise Any4Error("one table for the whole matrix comes with bf16 and groups of 128")
        _launch("any4_dequant_single_table", codes.device, pc, pl, ps, po, N, K, bits, pw)
    elif dt == torch.float16:
        if group != GROUP:
            raise Any4Error("fp16 inputs come with groups of 128")
        _launch("any4_dequant_f16", codes.device, pc, pl, ps, po, N, K, bits, pw)
    elif group == GROUP:
        _launch("any4_dequant", codes.device, pc, pl, ps, po, N, K, bits, pw)
    else:
        _launch("any4_dequant_grouped", codes.device, pc, pl, ps, po, N, K, bits, group, pw)
    return out


def _gemm(entry: str, x, codes, N, lut, scale, offset, bits, out, workspace, group=None):
    """the checked call, one argument after the other: what the native call below says no to comes here to be named"""
    M, K = x.shape
    dt = x.dtype if isinstance(x, torch.Tensor) and x.dtype == torch.float16 else torch.bfloat16
    if dt == torch.float16:
        if entry != "any4_gemm":
            raise Any4Error("fp16 inputs come with groups of 128 and the plain code layout")
        entry = "any4_gemm_f16"
    px = _dev(x, dt, "x")
    pc = _dev(codes, torch.int32, "codes")
    # a table of ONE row for a matrix of several: the single-table formats (any4_gemm_single_table)
    single = lut is not None and N != 1 and tuple(lut.shape) == (1, 1 << bits)
    if single:
        if entry != "any4_gemm":
            raise Any4Error("one table for the whole matrix comes with bf16, groups of 128 and the plain code layout")
        entry = "any4_gemm_single_table"
    _check_quant_shapes(codes, lut, scale, offset, N, K, bits, GROUP if group is None else group,
                        repacked=entry == "any4_gemm_repacked", single_table=single)
    pl = _dev(lut, dt, "lut") if lut is not None else None
    ps = _dev(scale, dt, "scale")
    po = _dev(offset, dt, "offset")
    if out is None:
        out = torch.empty((M, N), dtype=dt, device=x.device)
    _shape(out, (M, N), "out")
    py = _dev(out, dt, "out")
    need = _bytes_on(x.device, "any4_gemm_workspace_bytes", M, N, K, bits)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    pw, wbytes = _scratch(workspace, x.device) if workspace is not None else (None, 0)
    if group is None:
        _launch(entry, x.device, px, pc, pl, ps, po, M, N, K, bits, py, pw, wbytes)
    else:
        _launch(entry, x.device, px, pc, pl, ps, po, M, N, K, bits, group, py, pw, wbytes)
    return out


def _native(x, codes, lut, scale, offset, bits, out, workspace, group, repacked):
    """a plain valid call in native code (csrc/any4_torch.cpp): the output, or None with nothing done"""
    if _native_gemm is None:
        load_library()
    r = _native_gemm(x, codes, lut, scale, offset, bits, out, workspace, group, repacked)
    if r.__class__ is int:
        _check(r, "any4_gemm_repacked" if repacked else "any4_gemm")
    return r


def any4_gemm(x: torch.Tensor, codes: torch.Tensor, lut: torch.Tensor | None, scale: torch.Tensor,
              offset: torch.Tensor, bits: int = 4, out: torch.Tensor | None = None,
              workspace: torch.Tensor | None = None, group: int = GROUP) -> torch.Tensor:
    """bf16 [M,N] = x[M,K] . dequant(codes, lut, scale, offset)[N,K]^T
    (lut None with bits 4: the int4 grid, value = code - 8, run without a table; lut of shape
    [1, 2^bits]: one table for the whole matrix, any4_gemm_single_table);
    scale / offset are [N, K / group] (any4_gemm_grouped when group is not 128).
    With x, lut, scale, offset all fp16 the result is fp16 (any4_gemm_f16: groups of 128, a table)."""
    r = _native(x, codes, lut, scale, offset, bits, out, workspace, group, False)
    if r is not None:
        return r
    if group == GROUP:
        return _gemm("any4_gemm", x, codes, codes.shape[0], lut, scale, offset, bits, out, workspace)
    return _gemm("any4_gemm_grouped", x, codes, codes.shape[0], lut, scale, offset, bits, out, workspace, group)


NOALLOC_SCRATCH_BYTES = 48 << 20


def any4_gemm_noalloc(x: torch.Tensor, codes: torch.Tensor, lut: torch.Tensor | None, scale: torch.Tensor,
                      offset: torch.Tensor, bits: int = 4, out: torch.Tensor | None = None) -> torch.Tensor:
    """any4_gemm without a workspace: the library's own fixed scratch array serves (see include/any4.h;
    calls on one GPU must not overlap in time).  `out` should be passed by callers that must not allocate."""
    M, K = x.shape
    N = codes.shape[0]
    px = _dev(x, torch.bfloat16, "x")
    pc = _dev(codes, torch.int32, "codes")
    _check_quant_shapes(codes, lut, scale, offset, N, K, bits, GROUP)
    pl = _dev(lut, torch.bfloat16, "lut") if lut is not None else None
    ps = _dev(scale, torch.bfloat16, "scale")
    po = _dev(offset, torch.bfloat16, "offset")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    _shape(out, (M, N), "out")
    py = _dev(out, torch.bfloat16, "out")
    _launch("any4_gemm_noalloc", x.device, px, pc, pl, ps, po, M, N, K, bits, py)
    return out


def any4_repack_bytes(N: int, K: int, bits: int = 4) -> int:
    return int(load_library().any4_repack_bytes(N, K, bits))


def any4_repack(codes: torch.Tensor, bits: int = 4) -> torch.Tensor:
    """int32 [N, K*bits/32] packed codes -> the tile-major layout any4_gemm_repacked reads
    (int32, flat, any4_repack_bytes(N, K, bits) bytes)."""
    lib = load_library()
    N, W = codes.shape
    K = W * 32 // bits
    pc = _dev(codes, torch.int32, "codes")
    nbytes = int(lib.any4_repack_bytes(N, K, bits))
    if nbytes == 0:
        raise Any4Error("any4_repack: bad shape or bits")
    out = torch.empty(nbytes // 4, dtype=torch.int32, device=codes.device)
    _launch("any4_repack", codes.device, pc, N, K, bits, out.data_ptr())
    return out


def any4_gemm_repacked(x: torch.Tensor, rcodes: torch.Tensor, lut: torch.Tensor, scale: torch.Tensor,
                       offset: torch.Tensor, bits: int = 4, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """any4_gemm on codes re-arranged by any4_repack; N is taken from scale."""
    r = _native(x, rcodes, lut, scale, offset, bits, out, workspace, GROUP, True)
    if r is not None:
        return r
    return _gemm("any4_gemm_repacked", x, rcodes, scale.shape[0], lut, scale, offset, bits, out, workspace)


def any4_quantize_max_k() -> int:
    return int(load_library().any4_quantize_max_k())


def any4_quantize(w: torch.Tensor, act: torch.Tensor | None, u: torch.Tensor, bits: int = 4,
                  symmetric: bool = False, iters: int = 20, centre_gap: float | None = None):
    """fp32 [N,K] weights, fp32 [K] mean |activation| per channel (or None), fp32 [N, 2^bits]
    uniform draws -> dict with codes_u8 uint8 [N,K], lut bf16 [N,2^bits], scale / offset bf16
    [N,K/128] and msteps int32 [N].  Everything stays in device memory.  centre_gap: None calls
    any4_quantize, a number calls any4_quantize_with_gap."""
    N, K = w.shape
    L = 1 << bits
    pw = _dev(w, torch.float32, "w")
    pa = _dev(act, torch.float32, "act") if act is not None else None
    if tuple(u.shape) != (N, L):
        raise Any4Error(f"u must have shape ({N}, {L})")
    pu = _dev(u, torch.float32, "u")
    dev = w.device
    codes = torch.empty((N, K), dtype=torch.uint8, device=dev)
    lut = torch.empty((N, L), dtype=torch.bfloat16, device=dev)
    scale = torch.empty((N, max(K // GROUP, 0)), dtype=torch.bfloat16, device=dev)
    offset = torch.empty((N, max(K // GROUP, 0)), dtype=torch.bfloat16, device=dev)
    msteps = torch.empty((N,), dtype=torch.int32, device=dev)
    if centre_gap is None:
        _launch("any4_quantize", dev, pw, pa, pu, N, K, bits, int(symmetric), iters, codes.data_ptr(), lut.data_ptr(),
                scale.data_ptr(), offset.data_ptr(), msteps.data_ptr())
    else:
        _launch("any4_quantize_with_gap", dev, pw, pa, pu, N, K, bits, int(symmetric), iters, float(centre_gap),
                codes.data_ptr(), lut.data_ptr(), scale.data_ptr(), offset.data_ptr(), msteps.data_ptr())
    return {"codes_u8": codes, "lut": lut, "scale": scale, "offset": offset, "msteps": msteps}


# The key-value cache and the attention over it

def any4_kv_cache(pages: int, kv_heads: int, head_dim: int, page_size: int = 64, bits: int = 16, dtype: torch.dtype = torch.bfloat16,
                  device="cuda"):
    """(cache_k, cache_v, scales) of a paged cache, zeros: [pages, kv_heads, page_size, head_dim] of dtype with 16 bits, with 8 and 4
    bits codes (uint8, two to a byte with 4) and bf16 scales [pages, kv_heads, page_size, 4]; scales is None with 16 bits."""
    if bits not in (16, 8, 4):
        raise Any4Error(f"bits must be 16, 8 or 4, got {bits}")
    shape = (pages, kv_heads, page_size, head_dim if bits == 16 else head_dim * bits // 8)
    k, v = (torch.zeros(shape, dtype=dtype if bits == 16 else torch.uint8, device=device) for _ in range(2))
    return k, v, None if bits == 16 else torch.zeros((pages, kv_heads, page_size, 4), dtype=torch.bfloat16, device=device)


def _rows(t, dtype, name: str, shape) -> tuple[int, int, int]:
    """address and strides of rows [tokens, heads, head_dim]: a head's values side by side, the rest as it comes"""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise Any4Error(f"{name} must be a tensor in device memory")
    if t.dtype != dtype:
        raise Any4Error(f"{name} must have dtype {dtype}, got {t.dtype}")
    _shape(t, shape, name)
    if t.stride(2) != 1:
        raise Any4Error(f"{name}: the values of a head must lie side by side")
    return t.data_ptr(), t.stride(0), t.stride(1)


def _same_device(first, *others) -> None:
    for t in others:
        if t is not None and t.device != first.device:
            raise Any4Error(f"all tensors must be on one device, got {first.device} and {t.device}")


def _cache(cache_k, cache_v, scales, bits: int, dtype) -> tuple[_KvCache, int, int]:
    """the C structure, KV heads and head_dim"""
    if bits not in (16, 8, 4):
        raise Any4Error(f"bits must be 16, 8 or 4, got {bits}")
    if dtype not in (torch.bfloat16, torch.float16):
        raise Any4Error(f"the 16-bit values must be bf16 or fp16, got {dtype}")
    if not isinstance(cache_k, torch.Tensor) or cache_k.dim() != 4:
        raise Any4Error("cache_k must be a tensor of 4 dimensions: pages, kv_heads, page_size, head_dim (codes: bytes)")
    held = dtype if bits == 16 else torch.uint8
    pk, pv = _dev(cache_k, held, "cache_k"), _dev(cache_v, held, "cache_v")
    _shape(cache_v, cache_k.shape, "cache_v")
    pages, heads, page, width = cache_k.shape
    ps = None
    if bits != 16:
        ps = _dev(scales, torch.bfloat16, "scales")
        _shape(scales, (pages, heads, page, 4), "scales")
    _same_device(cache_k, cache_v, scales if bits != 16 else None)
    dim = width if bits == 16 else width * 8 // bits
    return _KvCache(pk, pv, ps, pages, page, heads, dim, bits, int(dtype == torch.float16)), heads, dim


def any4_kv_write(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor,
                  scales: torch.Tensor | None = None, bits: int = 16) -> None:
    """k, v [tokens, kv_heads, head_dim] (bf16 or fp16; slices of a fused projection's rows serve as they are) into slots
    (int64 [tokens]; a slot outside the cache leaves its token out) of the cache, with 8 and 4 bits quantised on the way."""
    r = _calls().kv_write(k, v, slots, cache_k, cache_v, scales, bits)
    if r is not None:
        if r.__class__ is int:
            _check(r, "any4_kv_write")
        return
    if not isinstance(k, torch.Tensor):
        raise Any4Error("k must be a tensor in device memory")
    cache, heads, dim = _cache(cache_k, cache_v, scales, bits, k.dtype)
    shape = (slots.shape[0] if isinstance(slots, torch.Tensor) and slots.dim() == 1 else -1, heads, dim)
    ptr = _dev(slots, torch.int64, "slots")
    if shape[0] < 0:
        raise Any4Error("slots must have one dimension")
    pk, pv = _rows(k, k.dtype, "k", shape), _rows(v, k.dtype, "v", shape)
    _same_device(k, v, slots, cache_k)
    _launch("any4_kv_write", cache_k.device, *pk, *pv, shape[0], ptr, ctypes.byref(cache))


def any4_kv_read(cache_k: torch.Tensor, cache_v: torch.Tensor, slots: torch.Tensor, scales: torch.Tensor | None = None, bits: int = 16,
                 dtype: torch.dtype = torch.bfloat16, out: tuple[torch.Tensor, torch.Tensor] | None = None):
    """(k, v) [tokens, kv_heads, head_dim] of slots (int64 [tokens]) of the cache, in dtype (the cache's own with 16 bits); zeros
    for a slot outside the cache."""
    try:
        out_k, out_v = (None, None) if out is None else out
    except (TypeError, ValueError):
        raise Any4Error("out must be a pair of tensors, k and v") from None
    if dtype is torch.bfloat16 or dtype is torch.float16:
        r = _calls().kv_read(cache_k, cache_v, slots, scales, bits, dtype is torch.float16, out_k, out_v)
        if r is not None:
            if r.__class__ is int:
                _check(r, "any4_kv_read")
            return r
    cache, heads, dim = _cache(cache_k, cache_v, scales, bits, dtype)
    ptr = _dev(slots, torch.int64, "slots")
    if slots.dim() != 1:
        raise Any4Error("slots must have one dimension")
    n = slots.shape[0]
    k, v = (out_k, out_v) if out is not None else (torch.empty((n, heads, dim), dtype=dtype, device=cache_k.device) for _ in range(2))
    pk, pv = _dev(k, dtype, "out[0]"), _dev(v, dtype, "out[1]")
    _shape(k, (n, heads, dim), "out[0]")
    _shape(v, (n, heads, dim), "out[1]")
    _same_device(cache_k, slots, k, v)
    _launch("any4_kv_read", cache_k.device, ctypes.byref(cache), ptr, n, pk, pv)
    return k, v


def any4_attn_decode_workspace_bytes(requests: int, heads: int, kv_heads: int, head_dim: int, max_tokens: int) -> int:
    return int(load_library().any4_attn_decode_workspace_bytes(requests, heads, kv_heads, head_dim, max_tokens))


def any4_attn_decode(q: torch.Tensor, cache_k: torch.Tensor, cache_v: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                     scales: torch.Tensor | None = None, bits: int = 16, softmax_scale: float | None = None,
                     out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """[requests, heads, head_dim]: the newest token of each request (q, of that shape; slices of a fused projection's rows serve as
    they are) attends to the first lengths[r] (int32 [requests]) tokens of its pages (page_table, int32 [requests, table_width]) in
    the cache.  Query head h reads KV head h // (heads // kv_heads); softmax_scale is head_dim ** -0.5 unless given."""
    r = _calls().attn_decode(q, cache_k, cache_v, page_table, lengths, scales, bits, softmax_scale, out, workspace)
    if r is not None:
        if r.__class__ is int:
            _check(r, "any4_attn_decode")
        return r
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise Any4Error("q must be a tensor of 3 dimensions: requests, heads, head_dim")
    n, heads = q.shape[:2]
    cache, kv_heads, dim = _cache(cache_k, cache_v, scales, bits, q.dtype)
    pq = _rows(q, q.dtype, "q", (n, heads, dim))
    if heads < 1 or kv_heads < 1 or heads % kv_heads:
        raise Any4Error(f"{heads} query heads are no multiple of {kv_heads} KV heads")
    if not isinstance(page_table, torch.Tensor) or not page_table.is_cuda or page_table.dtype != torch.int32:
        raise Any4Error("page_table must be an int32 tensor in device memory")
    if page_table.dim() != 2 or page_table.shape[0] != n or page_table.stride(1) != 1:
        raise Any4Error(f"page_table must have {n} rows of page numbers that lie side by side, got shape {tuple(page_table.shape)}")
    pl = _dev(lengths, torch.int32, "lengths")
    _shape(lengths, (n,), "lengths")
    if out is None:
        out = torch.empty((n, heads, dim), dtype=q.dtype, device=q.device)
    _shape(out, (n, heads, dim), "out")
    po = _dev(out, q.dtype, "out")
    _same_device(q, cache_k, page_table, lengths, out)
    width = page_table.shape[1]
    need = _bytes_on(q.device, "any4_attn_decode_workspace_bytes", n, heads, kv_heads, dim, width * cache.page_size)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    pw, wbytes = _scratch(workspace, q.device) if workspace is not None else (None, 0)
    _launch("any4_attn_decode", q.device, *pq, ctypes.byref(cache), page_table.data_ptr(), page_table.stride(0), width, pl, n, heads,
            dim ** -0.5 if softmax_scale is None else softmax_scale, po, pw, wbytes)
    return out


def any4_attn_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_starts: torch.Tensor, k_starts: torch.Tensor | None = None,
                     causal: bool = True, softmax_scale: float | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """[q_tokens, heads, head_dim]: packed prompts, request r in rows q_starts[r] .. q_starts[r + 1] - 1 of q and k_starts[r] .. of k and v
    [k_tokens, kv_heads, head_dim] (int32 [requests + 1]; k_starts None: q_starts).  Where a request has more rows in k, the first
    of them are the context in front of its queries: causal, query i of nq sees keys 0 .. i + nk - nq."""
    r = _calls().attn_prompt(q, k, v, q_starts, k_starts, causal, softmax_scale, out)
    if r is not None:
        if r.__class__ is int:
            _check(r, "any4_attn_prompt")
        return r
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise Any4Error(f"{name} must be a tensor of 3 dimensions: tokens, heads, head_dim")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise Any4Error(f"q must be bf16 or fp16, got {q.dtype}")
    n, heads, dim = q.shape
    kv_heads = k.shape[1]
    if heads < 1 or kv_heads < 1 or heads % kv_heads:
        raise Any4Error(f"{heads} query heads are no multiple of {kv_heads} KV heads")
    pq, pk, pv = _rows(q, q.dtype, "q", q.shape), _rows(k, q.dtype, "k", (k.shape[0], kv_heads, dim)), _rows(v, q.dtype, "v", (k.shape[0], kv_heads, dim))
    ps = _dev(q_starts, torch.int32, "q_starts")
    if q_starts.dim() != 1 or q_starts.shape[0] < 1:
        raise Any4Error("q_starts must have one entry for each request and one more")
    if k_starts is None:
        if k.shape[0] != n:
            raise Any4Error(f"without k_starts k has as many rows as q, {n}, got {k.shape[0]}")
        k_starts = q_starts
    pt = _dev(k_starts, torch.int32, "k_starts")
    _shape(k_starts, q_starts.shape, "k_starts")
    if out is None:
        out = torch.empty((n, heads, dim), dtype=q.dtype, device=q.device)
    _shape(out, (n, heads, dim), "out")
    po = _dev(out, q.dtype, "out")
    _same_device(q, k, v, q_starts, k_starts, out)
    _launch("any4_attn_prompt", q.device, *pq, *pk, *pv, n, k.shape[0], ps, pt, q_starts.shape[0] - 1, heads, kv_heads, dim,
            int(q.dtype == torch.float16), int(causal), dim ** -0.5 if softmax_scale is None else softmax_scale, po)
    return out
