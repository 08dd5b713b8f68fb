// The GEMM, cache and attention entry points of binding.py for the ordinary, valid call, in native code.
//
// A decode-size GEMM takes the GPU 5 - 10 us; checking shapes and types, asking for the workspace size,
// allocating the output and calling through ctypes took the host 13 us in Python, so that one call after
// another was bound by the host (1 x 1024 x 1024: 13.2 us a call, 4.7 us of it on the GPU).  gemm() does
// the same checks on the tensors themselves and calls the C ABI.  It only ever says yes: whatever is not a
// plain valid call (a wrong type, shape, device, layout, a combination that does not exist) returns None
// with nothing done, and binding.py goes through its own checks, which name the mistake.  The functions for the cache and for
// attention are the same for calls whose kernels take 3 - 5 us.  All of them run on the tensors' device, on torch's current stream of
// it, and without the interpreter's lock while they launch (a full queue makes a launch wait).
#include "any4_torch.h"

using namespace any4_torch;

namespace any4_torch {

// torch's current stream of the tensors' device, which is the current one for as long as the guard lives.  (The stream says which device is
// current: a guard that is not needed took 0.25 us of a call of 5.)
void* stream_on(const c10::Device& device, c10::OptionalDeviceGuard& guard) {
    c10::hip::HIPStream s = c10::hip::getCurrentHIPStream();
    if (s.device_index() != device.index()) {
        guard.reset_device(device);
        s = c10::hip::getCurrentHIPStream();
    }
    return s.stream();
}

}  // namespace any4_torch

namespace {

// gemm(x, codes, lut, scale, offset, bits, out, workspace, group, repacked)
//   -> the output tensor; None: not a plain valid call, nothing was done; an int: the runtime refused a launch
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS                                               // out of device memory and the like, as torch raises it
    if (n != 10) Py_RETURN_NONE;
    const at::Tensor *x = tensor(a[0]), *codes = tensor(a[1]), *scale = tensor(a[3]), *offset = tensor(a[4]);
    const bool has_lut = a[2] != Py_None, has_out = a[6] != Py_None, has_ws = a[7] != Py_None;
    const at::Tensor *lut = has_lut ? tensor(a[2]) : nullptr, *out = has_out ? tensor(a[6]) : nullptr,
                     *ws = has_ws ? tensor(a[7]) : nullptr;
    if (!x || !codes || !scale || !offset || (has_lut && !lut) || (has_out && !out) || (has_ws && !ws)) Py_RETURN_NONE;
    if (!PyLong_CheckExact(a[5]) || !PyLong_CheckExact(a[8])) Py_RETURN_NONE;
    const long bits = PyLong_AsLong(a[5]), group = PyLong_AsLong(a[8]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const bool repacked = a[9] == Py_True;
    if (x->dim() != 2 || codes->dim() < 1 || scale->dim() != 2) Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1), N = repacked ? scale->size(0) : codes->size(0);
    const at::ScalarType ty = x->scalar_type();
    const bool f16 = ty == at::kHalf;
    if (!f16 && ty != at::kBFloat16) Py_RETURN_NONE;
    if (bits < 2 || bits > 4 || M < 1 || N < 1 || K < 1 || K % ANY4_GROUP || group < 1 || K % group) Py_RETURN_NONE;
    if (!plain(*x, ty) || !plain(*codes, at::kInt) || !plain(*scale, ty) || !plain(*offset, ty)) Py_RETURN_NONE;
    const int64_t words = K * bits / 32, L = (int64_t)1 << bits;
    if (repacked ? codes->numel() != (N + 15) / 16 * 16 * words : !shaped(*codes, N, words)) Py_RETURN_NONE;
    if (!shaped(*scale, N, K / group) || !shaped(*offset, N, K / group)) Py_RETURN_NONE;
    bool one_table = false;
    if (lut) {
        if (!plain(*lut, ty)) Py_RETURN_NONE;
        one_table = N != 1 && shaped(*lut, 1, L);
        if (!one_table && !shaped(*lut, N, L)) Py_RETURN_NONE;
    }
    if ((f16 || one_table || repacked) && group != ANY4_GROUP) Py_RETURN_NONE;
    if ((f16 && (one_table || repacked)) || (one_table && repacked)) Py_RETURN_NONE;
    if (out && !(plain(*out, ty) && shaped(*out, M, N))) Py_RETURN_NONE;
    // (of any type, but as much memory as it has elements, and on the device)
    if (ws && !(ws->layout() == at::kStrided && ws->device() == x->device() && ws->is_non_overlapping_and_dense())) Py_RETURN_NONE;

    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(x->device(), guard);
    at::Tensor y = out ? *out : at::empty({M, N}, x->options().requires_grad(false));
    at::Tensor scratch;
    void* wp = nullptr;
    size_t wbytes = 0;
    if (ws) {
        wp = ws->data_ptr();
        wbytes = (size_t)ws->numel() * ws->element_size();
    } else if (const size_t need = any4_gemm_workspace_bytes(M, N, K, (int)bits)) {
        scratch = at::empty({(int64_t)need}, x->options().dtype(at::kByte).requires_grad(false));
        wp = scratch.data_ptr();
        wbytes = need;
    }
    const uint16_t *px = u16(*x), *pl = lut ? u16(*lut) : nullptr, *ps = u16(*scale), *po = u16(*offset);
    const uint32_t* pc = static_cast<const uint32_t*>(codes->data_ptr());
    uint16_t* py = static_cast<uint16_t*>(y.data_ptr());
    const int b = (int)bits;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (repacked) rc = any4_gemm_repacked(px, pc, pl, ps, po, M, N, K, b, py, wp, wbytes, stream);
    else if (f16) rc = any4_gemm_f16(px, pc, pl, ps, po, M, N, K, b, py, wp, wbytes, stream);
    else if (one_table) rc = any4_gemm_single_table(px, pc, pl, ps, po, M, N, K, b, py, wp, wbytes, stream);
    else if (group == ANY4_GROUP) rc = any4_gemm(px, pc, pl, ps, po, M, N, K, b, py, wp, wbytes, stream);
    else rc = any4_gemm_grouped(px, pc, pl, ps, po, M, N, K, b, (int)group, py, wp, wbytes, stream);
    Py_END_ALLOW_THREADS
    if (rc == ANY4_ERR_HIP) return PyLong_FromLong(rc);
    if (rc != ANY4_OK) Py_RETURN_NONE;                             // refused before any launch: binding.py names the call and the mistake
    if (out) { Py_INCREF(a[6]); return a[6]; }
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

// kv_write(k, v, slots, cache_k, cache_v, scales, bits) -> True; None and an int as gemm's
PyObject* kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7) Py_RETURN_NONE;
    const at::Tensor *k = tensor(a[0]), *v = tensor(a[1]), *slots = tensor(a[2]), *ck = tensor(a[3]), *cv = tensor(a[4]), *scales;
    long bits;
    any4_kv_cache c;
    if (!k || !v || !slots || !ck || !cv || !optional_tensor(a[5], scales) || !whole(a[6], bits)) Py_RETURN_NONE;
    if (!kv_cache(*ck, *cv, scales, bits, k->scalar_type(), c) || !list(*slots, at::kLong, *ck)) Py_RETURN_NONE;
    const int64_t tokens = slots->size(0);
    if (!rows(*k, k->scalar_type(), tokens, c.kv_heads, c.head_dim, *ck) || !rows(*v, k->scalar_type(), tokens, c.kv_heads, c.head_dim, *ck)) Py_RETURN_NONE;
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(ck->device(), guard);
    const Rows kr(*k), vr(*v);
    const int64_t* ps = static_cast<const int64_t*>(slots->data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_kv_write(kr.p, kr.token, kr.head, vr.p, vr.token, vr.head, tokens, ps, &c, stream);
    Py_END_ALLOW_THREADS
    if (rc == ANY4_OK) Py_RETURN_TRUE;
    if (rc == ANY4_ERR_HIP) return PyLong_FromLong(rc);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// kv_read(cache_k, cache_v, slots, scales, bits, f16, out_k, out_v) -> (k, v)
PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    const at::Tensor *ck = tensor(a[0]), *cv = tensor(a[1]), *slots = tensor(a[2]), *scales, *ok, *ov;
    long bits;
    any4_kv_cache c;
    const at::ScalarType ty = a[5] == Py_True ? at::kHalf : at::kBFloat16;
    if (!ck || !cv || !slots || !optional_tensor(a[3], scales) || !whole(a[4], bits) || !optional_tensor(a[6], ok) || !optional_tensor(a[7], ov)) Py_RETURN_NONE;
    if (!ok != !ov || !kv_cache(*ck, *cv, scales, bits, ty, c) || !list(*slots, at::kLong, *ck)) Py_RETURN_NONE;
    const int64_t tokens = slots->size(0);
    for (const at::Tensor* o : {ok, ov})
        if (o && !(plain(*o, ty) && o->dim() == 3 && o->size(0) == tokens && o->size(1) == c.kv_heads && o->size(2) == c.head_dim && o->device() == ck->device())) Py_RETURN_NONE;
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(ck->device(), guard);
    at::Tensor k = ok ? *ok : at::empty({tokens, c.kv_heads, c.head_dim}, ck->options().dtype(ty).requires_grad(false));
    at::Tensor v = ov ? *ov : at::empty({tokens, c.kv_heads, c.head_dim}, ck->options().dtype(ty).requires_grad(false));
    const int64_t* ps = static_cast<const int64_t*>(slots->data_ptr());
    uint16_t *pk = static_cast<uint16_t*>(k.data_ptr()), *pv = static_cast<uint16_t*>(v.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_kv_read(&c, ps, tokens, pk, pv, stream);
    Py_END_ALLOW_THREADS
    if (rc == ANY4_ERR_HIP) return PyLong_FromLong(rc);
    if (rc != ANY4_OK) Py_RETURN_NONE;
    PyObject* both = PyTuple_New(2);
    if (!both) return nullptr;
    PyTuple_SET_ITEM(both, 0, answer(rc, a[6], std::move(k)));
    PyTuple_SET_ITEM(both, 1, answer(rc, a[7], std::move(v)));
    return both;
    END_HANDLE_TH_ERRORS
}

// attn_decode(q, cache_k, cache_v, page_table, lengths, scales, bits, softmax_scale, out, workspace)
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *ck = tensor(a[1]), *cv = tensor(a[2]), *table = tensor(a[3]), *lengths = tensor(a[4]), *scales, *out, *ws;
    long bits;
    float scale;
    any4_kv_cache c;
    if (!q || !ck || !cv || !table || !lengths || !optional_tensor(a[5], scales) || !whole(a[6], bits) || !optional_tensor(a[8], out) ||
        !optional_tensor(a[9], ws) || q->dim() != 3)
        Py_RETURN_NONE;
    const at::ScalarType ty = q->scalar_type();
    const int64_t requests = q->size(0), heads = q->size(1);
    if (!kv_cache(*ck, *cv, scales, bits, ty, c) || !rows(*q, ty, requests, heads, c.head_dim, *ck) || !scale_of(a[7], c.head_dim, scale)) Py_RETURN_NONE;
    if (heads < 1 || heads > 0xFFFF || c.kv_heads < 1 || heads % c.kv_heads) Py_RETURN_NONE;
    if (!list(*lengths, at::kInt, *ck) || lengths->size(0) != requests) Py_RETURN_NONE;
    if (!table->is_cuda() || table->scalar_type() != at::kInt || table->layout() != at::kStrided || table->dim() != 2 || table->size(0) != requests ||
        table->stride(1) != 1 || table->device() != ck->device())
        Py_RETURN_NONE;
    if (out && !(plain(*out, ty) && rows(*out, ty, requests, heads, c.head_dim, *ck))) Py_RETURN_NONE;
    if (ws && !(ws->layout() == at::kStrided && ws->device() == ck->device() && ws->is_non_overlapping_and_dense())) Py_RETURN_NONE;
    const int64_t width = table->size(1), table_stride = table->stride(0);
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(ck->device(), guard);
    at::Tensor o = out ? *out : at::empty({requests, heads, c.head_dim}, q->options().requires_grad(false));
    at::Tensor scratch;
    void* wp = nullptr;
    size_t wbytes = 0;
    if (ws) {
        wp = ws->data_ptr();
        wbytes = (size_t)ws->numel() * ws->element_size();
    } else if (const size_t need = any4_attn_decode_workspace_bytes(requests, (int)heads, c.kv_heads, c.head_dim, width * c.page_size)) {
        scratch = at::empty({(int64_t)need}, q->options().dtype(at::kByte).requires_grad(false));
        wp = scratch.data_ptr();
        wbytes = need;
    }
    const Rows qr(*q);
    const int32_t *pt = static_cast<const int32_t*>(table->data_ptr()), *pl = static_cast<const int32_t*>(lengths->data_ptr());
    uint16_t* po = static_cast<uint16_t*>(o.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_attn_decode(qr.p, qr.token, qr.head, &c, pt, table_stride, width, pl, requests, (int)heads, scale, po, wp, wbytes, stream);
    Py_END_ALLOW_THREADS
    return answer(rc, a[8], std::move(o));
    END_HANDLE_TH_ERRORS
}

// attn_prompt(q, k, v, q_starts, k_starts, causal, softmax_scale, out)
PyObject* attn_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *qs = tensor(a[3]), *ks, *out;
    float scale;
    if (!q || !k || !v || !qs || !optional_tensor(a[4], ks) || !optional_tensor(a[7], out) || q->dim() != 3 || k->dim() != 3) Py_RETURN_NONE;
    if (a[5] != Py_True && a[5] != Py_False) Py_RETURN_NONE;
    const at::ScalarType ty = q->scalar_type();
    if (ty != at::kBFloat16 && ty != at::kHalf) Py_RETURN_NONE;
    const int64_t nq = q->size(0), heads = q->size(1), dim = q->size(2), nk = k->size(0), kv_heads = k->size(1);
    if (heads < 1 || heads > 0xFFFF || kv_heads < 1 || kv_heads > 0xFFFF || heads % kv_heads || dim > 0xFFFF) Py_RETURN_NONE;
    if (!rows(*q, ty, nq, heads, dim, *q) || !rows(*k, ty, nk, kv_heads, dim, *q) || !rows(*v, ty, nk, kv_heads, dim, *q)) Py_RETURN_NONE;
    if (!list(*qs, at::kInt, *q) || qs->size(0) < 1 || (ks && (!list(*ks, at::kInt, *q) || ks->size(0) != qs->size(0)))) Py_RETURN_NONE;
    if ((!ks && nk != nq) || !scale_of(a[6], dim, scale)) Py_RETURN_NONE;
    if (out && !(plain(*out, ty) && rows(*out, ty, nq, heads, dim, *q))) Py_RETURN_NONE;
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(q->device(), guard);
    at::Tensor o = out ? *out : at::empty({nq, heads, dim}, q->options().requires_grad(false));
    const Rows qr(*q), kr(*k), vr(*v);
    const int32_t *pqs = static_cast<const int32_t*>(qs->data_ptr()), *pks = static_cast<const int32_t*>((ks ? ks : qs)->data_ptr());
    const int64_t requests = qs->size(0) - 1;
    const bool causal = a[5] == Py_True;
    uint16_t* po = static_cast<uint16_t*>(o.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_attn_prompt(qr.p, qr.token, qr.head, kr.p, kr.token, kr.head, vr.p, vr.token, vr.head, nq, nk, pqs, pks, requests, (int)heads, (int)kv_heads,
                          (int)dim, ty == at::kHalf, causal, scale, po, stream);
    Py_END_ALLOW_THREADS
    return answer(rc, a[7], std::move(o));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"kv_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_write)), METH_FASTCALL, "kv_write(k, v, slots, cache_k, cache_v, scales, bits)"},
    {"kv_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_read)), METH_FASTCALL,
     "kv_read(cache_k, cache_v, slots, scales, bits, f16, out_k, out_v)"},
    {"attn_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_decode)), METH_FASTCALL,
     "attn_decode(q, cache_k, cache_v, page_table, lengths, scales, bits, softmax_scale, out, workspace)"},
    {"attn_decode_window", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_decode_window)), METH_FASTCALL,
     "attn_decode_window(q, cache_k, cache_v, page_table, lengths, scales, bits, softmax_scale, out, workspace, window, sinks)"},
    {"attn_chunk", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_chunk)), METH_FASTCALL,
     "attn_chunk(q, cache_k, cache_v, page_table, q_starts, lengths, scales, bits, window, sinks, softmax_scale, out, workspace)"},
    {"attn_prompt_window", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_prompt_window)), METH_FASTCALL,
     "attn_prompt_window(q, k, v, q_starts, k_starts, window, sinks, softmax_scale, out)"},
    {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope)), METH_FASTCALL,
     "rope(q, k, positions, freqs, q_norm, k_norm, eps, interleaved, axis_of, out_q, out_k)"},
    {"rope_kv_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope_kv_write)), METH_FASTCALL,
     "rope_kv_write(q, k, v, positions, freqs, slots, cache_k, cache_v, scales, bits, q_norm, k_norm, eps, interleaved, axis_of, out, k_out)"},
    {"attn_prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_prompt)), METH_FASTCALL,
     "attn_prompt(q, k, v, q_starts, k_starts, causal, softmax_scale, out)"},
    {"gemm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gemm)), METH_FASTCALL,
     "gemm(x, codes, lut, scale, offset, bits, out, workspace, group, repacked)"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_any4_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__any4_torch(void) { return PyModule_Create(&module); }
