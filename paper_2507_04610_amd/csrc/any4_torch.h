// What the native calls of binding.py share: arguments as the C ABI takes them, the tensors' stream.
#pragma once
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <algorithm>
#include <cmath>
#include "any4.h"

namespace any4_torch {

inline const at::Tensor* tensor(PyObject* o) {
    return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
}
inline bool plain(const at::Tensor& t, at::ScalarType ty) {
    return t.is_cuda() && t.scalar_type() == ty && t.is_contiguous() && t.layout() == at::kStrided;
}
inline bool shaped(const at::Tensor& t, int64_t a, int64_t b) { return t.dim() == 2 && t.size(0) == a && t.size(1) == b; }

// torch's current stream of the tensors' device, which is the current one for as long as the guard lives
void* stream_on(const c10::Device& device, c10::OptionalDeviceGuard& guard);

inline const uint16_t* u16(const at::Tensor& t) { return static_cast<const uint16_t*>(t.data_ptr()); }

// The cache as the C ABI takes it, from tensors [pages, kv_heads, page_size, head_dim (bytes of codes)]; false: not a valid one
inline bool kv_cache(const at::Tensor& k, const at::Tensor& v, const at::Tensor* scales, long bits, at::ScalarType ty, any4_kv_cache& c) {
    const at::ScalarType held = bits == 16 ? ty : at::kByte;
    if ((bits != 16 && bits != 8 && bits != 4) || (ty != at::kBFloat16 && ty != at::kHalf) || k.dim() != 4) return false;
    if (!plain(k, held) || !plain(v, held) || v.sizes() != k.sizes() || v.device() != k.device()) return false;
    const int64_t pages = k.size(0), heads = k.size(1), page = k.size(2), width = k.size(3);
    if (heads > 0xFFFF || page > 0xFFFF || width > 0xFFFF) return false;
    c = any4_kv_cache{k.data_ptr(), v.data_ptr(), nullptr, pages, (int)page, (int)heads, (int)(bits == 16 ? width : width * 8 / bits), (int)bits, ty == at::kHalf};
    if (bits == 16) return true;
    if (!scales || !plain(*scales, at::kBFloat16) || scales->dim() != 4 || scales->size(0) != pages || scales->size(1) != heads ||
        scales->size(2) != page || scales->size(3) != 4 || scales->device() != k.device())
        return false;
    c.scales = static_cast<uint16_t*>(scales->data_ptr());
    return true;
}
// address and strides of rows [tokens, heads, head_dim]
struct Rows {
    const uint16_t* p;
    int64_t token, head;
    explicit Rows(const at::Tensor& t) : p(u16(t)), token(t.stride(0)), head(t.stride(1)) {}
};
// rows [tokens, heads, head_dim] whose heads' values lie side by side
inline bool rows(const at::Tensor& t, at::ScalarType ty, int64_t tokens, int64_t heads, int64_t dim, const at::Tensor& on) {
    return t.is_cuda() && t.scalar_type() == ty && t.layout() == at::kStrided && t.dim() == 3 && t.size(0) == tokens && t.size(1) == heads &&
           t.size(2) == dim && t.stride(2) == 1 && t.device() == on.device();
}
inline bool list(const at::Tensor& t, at::ScalarType ty, const at::Tensor& on) { return plain(t, ty) && t.dim() == 1 && t.device() == on.device(); }
// a tensor, or None; false: something else
inline bool optional_tensor(PyObject* o, const at::Tensor*& t) {
    t = o == Py_None ? nullptr : tensor(o);
    return o == Py_None || t;
}
inline bool whole(PyObject* o, long& v) {
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsLong(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}
// softmax_scale, or None: head_dim ** -0.5
inline bool scale_of(PyObject* o, int64_t dim, float& s) {
    if (o == Py_None) { s = (float)std::pow((double)dim, -0.5); return true; }
    if (!PyFloat_CheckExact(o)) return false;
    s = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
inline PyObject* answer(int rc, PyObject* given, at::Tensor&& made) {
    if (rc == ANY4_ERR_HIP) return PyLong_FromLong(rc);
    if (rc != ANY4_OK) Py_RETURN_NONE;
    if (given != Py_None) { Py_INCREF(given); return given; }
    return THPVariable_Wrap(std::move(made));
}

// the calls of any4_torch_rows.cpp
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* rope_kv_write(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* attn_decode_window(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* attn_chunk(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* attn_prompt_window(PyObject*, PyObject* const* a, Py_ssize_t n);

}  // namespace any4_torch
