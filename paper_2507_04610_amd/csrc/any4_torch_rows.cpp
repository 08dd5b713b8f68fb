// The entry points of binding.py for rotated rows, chunks and windows, for the ordinary, valid call: as those of any4_torch.cpp.
#include "any4_torch.h"

namespace any4_torch {

namespace {

// rows that can be written to: no value lies where another does
bool apart(const at::Tensor& t) {
    int64_t n1 = t.size(0), s1 = t.stride(0), n2 = t.size(1), s2 = t.stride(1);
    if (s1 < s2) { std::swap(n1, n2); std::swap(s1, s2); }
    if (n2 > 1 && s2 < t.size(2)) return false;
    return n1 <= 1 || s1 >= (n2 > 1 ? (n2 - 1) * s2 : 0) + t.size(2);
}
// positions [tokens] or [axes, tokens], freqs, q_norm, k_norm, eps, interleaved and axis_of of any4_rope; false: not valid ones
bool rotation(const at::Tensor* positions, const at::Tensor* freqs, const at::Tensor* q_norm, const at::Tensor* k_norm, PyObject* eps, PyObject* interleaved,
              const at::Tensor* axis_of, int64_t tokens, int64_t dim, at::ScalarType ty, const at::Tensor& on, any4_rotation& r) {
    if (!positions || !positions->is_cuda() || positions->scalar_type() != at::kLong || positions->layout() != at::kStrided || positions->device() != on.device()) return false;
    const int64_t d = positions->dim();
    if ((d != 1 && d != 2) || positions->size(d - 1) != tokens || (tokens > 1 && positions->stride(d - 1) != 1) || (d == 2 && (positions->size(0) < 1 || positions->size(0) > 4)))
        return false;
    if (!freqs || !list(*freqs, at::kDouble, on) || freqs->size(0) > dim / 2) return false;
    if (axis_of && (!list(*axis_of, at::kByte, on) || axis_of->size(0) != freqs->size(0))) return false;
    for (const at::Tensor* w : {q_norm, k_norm})
        if (w && (!list(*w, ty, on) || w->size(0) != dim)) return false;
    if (!PyFloat_CheckExact(eps) || (interleaved != Py_True && interleaved != Py_False)) return false;
    r = any4_rotation{static_cast<const int64_t*>(positions->data_ptr()), d == 2 ? positions->stride(0) : 0, static_cast<const double*>(freqs->data_ptr()),
                      axis_of ? static_cast<const uint8_t*>(axis_of->data_ptr()) : nullptr, q_norm ? u16(*q_norm) : nullptr, k_norm ? u16(*k_norm) : nullptr,
                      d == 2 ? (int)positions->size(0) : 1, (int)(2 * freqs->size(0)), interleaved == Py_True, (float)PyFloat_AS_DOUBLE(eps)};
    return true;
}

}  // namespace

// rope(q, k, positions, freqs, q_norm, k_norm, eps, interleaved, axis_of, out_q, out_k) -> (q, k)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 11) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *positions = tensor(a[2]), *freqs = tensor(a[3]), *qn, *kn, *axis_of, *oq, *ok;
    any4_rotation r;
    if (!q || !k || !optional_tensor(a[4], qn) || !optional_tensor(a[5], kn) || !optional_tensor(a[8], axis_of) || !optional_tensor(a[9], oq) ||
        !optional_tensor(a[10], ok) || q->dim() != 3 || k->dim() != 3)
        Py_RETURN_NONE;
    const at::ScalarType ty = q->scalar_type();
    if (ty != at::kBFloat16 && ty != at::kHalf) Py_RETURN_NONE;
    const int64_t tokens = q->size(0), heads = q->size(1), dim = q->size(2), kv_heads = k->size(1);
    if (heads < 1 || heads > 0xFFFF || kv_heads < 1 || kv_heads > 0xFFFF || dim > 0xFFFF) Py_RETURN_NONE;
    if (!rows(*q, ty, tokens, heads, dim, *q) || !rows(*k, ty, tokens, kv_heads, dim, *q)) Py_RETURN_NONE;
    if (!rotation(positions, freqs, qn, kn, a[6], a[7], axis_of, tokens, dim, ty, *q, r)) Py_RETURN_NONE;
    if ((oq && !(rows(*oq, ty, tokens, heads, dim, *q) && apart(*oq))) || (ok && !(rows(*ok, ty, tokens, kv_heads, dim, *q) && apart(*ok)))) Py_RETURN_NONE;
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(q->device(), guard);
    at::Tensor yq = oq ? *oq : at::empty({tokens, heads, dim}, q->options().requires_grad(false));
    at::Tensor yk = ok ? *ok : at::empty({tokens, kv_heads, dim}, q->options().requires_grad(false));
    const Rows qr(*q), kr(*k), yqr(yq), ykr(yk);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_rope(qr.p, qr.token, qr.head, kr.p, kr.token, kr.head, tokens, (int)heads, (int)kv_heads, (int)dim, ty == at::kHalf, &r,
                   const_cast<uint16_t*>(yqr.p), yqr.token, yqr.head, const_cast<uint16_t*>(ykr.p), ykr.token, ykr.head, stream);
    Py_END_ALLOW_THREADS
    if (rc == ANY4_ERR_HIP) return PyLong_FromLong(rc);
    if (rc != ANY4_OK) Py_RETURN_NONE;
    PyObject* both = PyTuple_New(2);
    if (!both) return nullptr;
    PyTuple_SET_ITEM(both, 0, answer(rc, a[9], std::move(yq)));
    PyTuple_SET_ITEM(both, 1, answer(rc, a[10], std::move(yk)));
    return both;
    END_HANDLE_TH_ERRORS
}

// rope_kv_write(q, k, v, positions, freqs, slots, cache_k, cache_v, scales, bits, q_norm, k_norm, eps, interleaved, axis_of, out, k_out) -> q
PyObject* rope_kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 17) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *positions = tensor(a[3]), *freqs = tensor(a[4]), *slots = tensor(a[5]),
                     *ck = tensor(a[6]), *cv = tensor(a[7]), *scales, *qn, *kn, *axis_of, *oq, *ok;
    long bits;
    any4_kv_cache c;
    any4_rotation r;
    if (!q || !k || !v || !slots || !ck || !cv || !optional_tensor(a[8], scales) || !whole(a[9], bits) || !optional_tensor(a[10], qn) || !optional_tensor(a[11], kn) ||
        !optional_tensor(a[14], axis_of) || !optional_tensor(a[15], oq) || !optional_tensor(a[16], ok) || q->dim() != 3)
        Py_RETURN_NONE;
    const at::ScalarType ty = q->scalar_type();
    if (!kv_cache(*ck, *cv, scales, bits, ty, c) || !list(*slots, at::kLong, *ck)) Py_RETURN_NONE;
    const int64_t tokens = slots->size(0), heads = q->size(1);
    if (heads < 1 || heads > 0xFFFF) Py_RETURN_NONE;
    if (!rows(*q, ty, tokens, heads, c.head_dim, *ck) || !rows(*k, ty, tokens, c.kv_heads, c.head_dim, *ck) || !rows(*v, ty, tokens, c.kv_heads, c.head_dim, *ck)) Py_RETURN_NONE;
    if (!rotation(positions, freqs, qn, kn, a[12], a[13], axis_of, tokens, c.head_dim, ty, *ck, r)) Py_RETURN_NONE;
    if ((oq && !(rows(*oq, ty, tokens, heads, c.head_dim, *ck) && apart(*oq))) || (ok && !(rows(*ok, ty, tokens, c.kv_heads, c.head_dim, *ck) && apart(*ok)))) Py_RETURN_NONE;
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(ck->device(), guard);
    at::Tensor yq = oq ? *oq : at::empty({tokens, heads, c.head_dim}, q->options().requires_grad(false));
    const Rows qr(*q), kr(*k), vr(*v), yqr(yq), ykr(ok ? *ok : *k);
    const int64_t* ps = static_cast<const int64_t*>(slots->data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_rope_kv_write(qr.p, qr.token, qr.head, kr.p, kr.token, kr.head, vr.p, vr.token, vr.head, tokens, (int)heads, &r, ps, &c,
                            const_cast<uint16_t*>(yqr.p), yqr.token, yqr.head, ok ? const_cast<uint16_t*>(ykr.p) : nullptr, ykr.token, ykr.head, stream);
    Py_END_ALLOW_THREADS
    return answer(rc, a[15], std::move(yq));
    END_HANDLE_TH_ERRORS
}

// attn_decode_window(q, cache_k, cache_v, page_table, lengths, scales, bits, softmax_scale, out, workspace, window, sinks)
PyObject* attn_decode_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *ck = tensor(a[1]), *cv = tensor(a[2]), *table = tensor(a[3]), *lengths = tensor(a[4]), *scales, *out, *ws;
    long bits, window, sinks;
    float scale;
    any4_kv_cache c;
    if (!q || !ck || !cv || !table || !lengths || !optional_tensor(a[5], scales) || !whole(a[6], bits) || !optional_tensor(a[8], out) ||
        !optional_tensor(a[9], ws) || !whole(a[10], window) || !whole(a[11], sinks) || q->dim() != 3)
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
    rc = any4_attn_decode_window(qr.p, qr.token, qr.head, &c, pt, table_stride, width, pl, requests, (int)heads, window, sinks, scale, po, wp, wbytes, stream);
    Py_END_ALLOW_THREADS
    return answer(rc, a[8], std::move(o));
    END_HANDLE_TH_ERRORS
}

// attn_chunk(q, cache_k, cache_v, page_table, q_starts, lengths, scales, bits, window, sinks, softmax_scale, out, workspace)
PyObject* attn_chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *ck = tensor(a[1]), *cv = tensor(a[2]), *table = tensor(a[3]), *starts = tensor(a[4]), *lengths = tensor(a[5]), *scales, *out, *ws;
    long bits, window, sinks;
    float scale;
    any4_kv_cache c;
    if (!q || !ck || !cv || !table || !starts || !lengths || !optional_tensor(a[6], scales) || !whole(a[7], bits) || !optional_tensor(a[11], out) ||
        !optional_tensor(a[12], ws) || !whole(a[8], window) || !whole(a[9], sinks) || q->dim() != 3)
        Py_RETURN_NONE;
    const at::ScalarType ty = q->scalar_type();
    const int64_t tokens = q->size(0), heads = q->size(1);
    if (!kv_cache(*ck, *cv, scales, bits, ty, c) || !rows(*q, ty, tokens, heads, c.head_dim, *ck) || !scale_of(a[10], c.head_dim, scale)) Py_RETURN_NONE;
    if (heads < 1 || heads > 0xFFFF || c.kv_heads < 1 || heads % c.kv_heads) Py_RETURN_NONE;
    if (!list(*lengths, at::kInt, *ck) || !list(*starts, at::kInt, *ck) || starts->size(0) != lengths->size(0) + 1) Py_RETURN_NONE;
    const int64_t requests = lengths->size(0);
    if (!table->is_cuda() || table->scalar_type() != at::kInt || table->layout() != at::kStrided || table->dim() != 2 || table->size(0) != requests ||
        table->stride(1) != 1 || table->device() != ck->device())
        Py_RETURN_NONE;
    if (out && !(plain(*out, ty) && rows(*out, ty, tokens, heads, c.head_dim, *ck))) Py_RETURN_NONE;
    if (ws && !(ws->layout() == at::kStrided && ws->device() == ck->device() && ws->is_non_overlapping_and_dense())) Py_RETURN_NONE;
    const int64_t width = table->size(1), table_stride = table->stride(0);
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(ck->device(), guard);
    at::Tensor o = out ? *out : at::empty({tokens, heads, c.head_dim}, q->options().requires_grad(false));
    at::Tensor scratch;
    void* wp = nullptr;
    size_t wbytes = 0;
    if (ws) {
        wp = ws->data_ptr();
        wbytes = (size_t)ws->numel() * ws->element_size();
    } else if (const size_t need = any4_attn_chunk_workspace_bytes(requests, tokens, (int)heads, c.kv_heads, c.head_dim, width * c.page_size)) {
        scratch = at::empty({(int64_t)need}, q->options().dtype(at::kByte).requires_grad(false));
        wp = scratch.data_ptr();
        wbytes = need;
    }
    const Rows qr(*q);
    const int32_t *pt = static_cast<const int32_t*>(table->data_ptr()), *ps = static_cast<const int32_t*>(starts->data_ptr()), *pl = static_cast<const int32_t*>(lengths->data_ptr());
    uint16_t* po = static_cast<uint16_t*>(o.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_attn_chunk(qr.p, qr.token, qr.head, &c, pt, table_stride, width, ps, pl, tokens, requests, (int)heads, window, sinks, scale, po, wp, wbytes, stream);
    Py_END_ALLOW_THREADS
    return answer(rc, a[11], std::move(o));
    END_HANDLE_TH_ERRORS
}

// attn_prompt_window(q, k, v, q_starts, k_starts, window, sinks, softmax_scale, out)
PyObject* attn_prompt_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *qs = tensor(a[3]), *ks, *out;
    float scale;
    long window, sinks;
    if (!q || !k || !v || !qs || !optional_tensor(a[4], ks) || !optional_tensor(a[8], out) || !whole(a[5], window) || !whole(a[6], sinks) || q->dim() != 3 || k->dim() != 3) Py_RETURN_NONE;
    const at::ScalarType ty = q->scalar_type();
    if (ty != at::kBFloat16 && ty != at::kHalf) Py_RETURN_NONE;
    const int64_t nq = q->size(0), heads = q->size(1), dim = q->size(2), nk = k->size(0), kv_heads = k->size(1);
    if (heads < 1 || heads > 0xFFFF || kv_heads < 1 || kv_heads > 0xFFFF || heads % kv_heads || dim > 0xFFFF) Py_RETURN_NONE;
    if (!rows(*q, ty, nq, heads, dim, *q) || !rows(*k, ty, nk, kv_heads, dim, *q) || !rows(*v, ty, nk, kv_heads, dim, *q)) Py_RETURN_NONE;
    if (!list(*qs, at::kInt, *q) || qs->size(0) < 1 || (ks && (!list(*ks, at::kInt, *q) || ks->size(0) != qs->size(0)))) Py_RETURN_NONE;
    if ((!ks && nk != nq) || !scale_of(a[7], dim, scale)) Py_RETURN_NONE;
    if (out && !(plain(*out, ty) && rows(*out, ty, nq, heads, dim, *q))) Py_RETURN_NONE;
    c10::OptionalDeviceGuard guard;
    void* const stream = stream_on(q->device(), guard);
    at::Tensor o = out ? *out : at::empty({nq, heads, dim}, q->options().requires_grad(false));
    const Rows qr(*q), kr(*k), vr(*v);
    const int32_t *pqs = static_cast<const int32_t*>(qs->data_ptr()), *pks = static_cast<const int32_t*>((ks ? ks : qs)->data_ptr());
    const int64_t requests = qs->size(0) - 1;
    uint16_t* po = static_cast<uint16_t*>(o.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = any4_attn_prompt_window(qr.p, qr.token, qr.head, kr.p, kr.token, kr.head, vr.p, vr.token, vr.head, nq, nk, pqs, pks, requests, (int)heads, (int)kv_heads,
                          (int)dim, ty == at::kHalf, window, sinks, scale, po, stream);
    Py_END_ALLOW_THREADS
    return answer(rc, a[8], std::move(o));
    END_HANDLE_TH_ERRORS
}

}  // namespace any4_torch
