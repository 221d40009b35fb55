// Marshalling for binding.py, for calls that are over in microseconds: checks that a call's tensors are what its description says and
// passes their addresses on.  Every function returns the library's return code, or None where a tensor is not as it has to be (binding.py
// then says which and why).  The same checks in Python took 2.4 us of a norm's 6.1 us per call (0.5 of 4.3 now; 3.9 are the launch's),
// 2.7 to 3.2 of a cache write or read's 6.9 and 7.4 (4.2 now).
#include <Python.h>
#include <string.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "moe355.h"

namespace {

// One call's arguments; `ok` falls where one of them is not as it has to be.
struct Args {
    PyObject* const* at;
    bool ok = true;

    template <typename F>
    F* function(int i) { return reinterpret_cast<F*>(PyLong_AsVoidPtr(at[i])); }

    // A description: a ctypes structure.
    template <typename C>
    C description(int i) {
        C c{};
        Py_buffer b;
        if (PyObject_GetBuffer(at[i], &b, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            ok = false;
            return c;
        }
        if (b.len == sizeof(C)) memcpy(&c, b.buf, sizeof(C));
        else ok = false;
        PyBuffer_Release(&b);
        return c;
    }
    const at::Tensor* tensor(int i) {
        if (at[i] == Py_None) return nullptr;
        if (!THPVariable_Check(at[i])) {
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(at[i]);
        if (!t.is_cuda()) ok = false;
        return &t;
    }
    // A contiguous device tensor of this type and size; None stays a null pointer (the library says whether it may be).
    void* array(int i, at::ScalarType type, int64_t numel) {
        const at::Tensor* t = tensor(i);
        if (t == nullptr) return nullptr;
        if (!ok || t->scalar_type() != type || t->numel() != numel || !t->is_contiguous()) {
            ok = false;
            return nullptr;
        }
        return t->data_ptr();
    }
    // [n, heads, dim] whose rows may be part of wider ones, each row contiguous.
    void* rows(int i, at::ScalarType type, int64_t n, int64_t heads, int64_t dim, int64_t* stride) {
        *stride = heads * dim;
        const at::Tensor* t = tensor(i);
        if (t == nullptr) return nullptr;
        ok = ok && t->scalar_type() == type && t->dim() == 3 && t->size(0) == n && t->size(1) == heads && t->size(2) == dim;
        if (!ok) return nullptr;
        if (n > 0 && (t->stride(2) != 1 || (t->stride(1) != dim && heads != 1))) ok = false;
        if (n > 1) *stride = t->stride(0);
        return t->data_ptr();
    }
    // A stream's handle, or the current stream of the current device for None; after all other arguments.
    void* stream(int i) { return !ok ? nullptr : at[i] == Py_None ? c10::hip::getCurrentHIPStream().stream() : PyLong_AsVoidPtr(at[i]); }

    at::ScalarType type(int32_t code) {
        if (code == MOE_F32) return at::kFloat;
        if (code == MOE_BF16) return at::kBFloat16;
        if (code != MOE_E4M3) ok = false;
        return at::kFloat8_e4m3fn;
    }
};

// The library's return code for good arguments, None for others, nothing with a Python exception.
template <typename Call>
PyObject* outcome(const Args& a, Call call) {
    if (PyErr_Occurred() != nullptr) return nullptr;
    if (!a.ok) Py_RETURN_NONE;
    PyThreadState* const thread = PyEval_SaveThread();
    const int rc = call();
    PyEval_RestoreThread(thread);
    return PyLong_FromLong(rc);
}

// No C++ exception passes into the interpreter's C code.
template <PyObject* (*F)(Args)>
PyObject* guarded(PyObject*, PyObject* const* at, Py_ssize_t n, Py_ssize_t wanted) {
    if (n != wanted) return PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", wanted, n);
    try {
        return F(Args{at});
    } catch (const std::exception& e) {
        return PyErr_Format(PyExc_RuntimeError, "%s", e.what());
    }
}

// (function, -, cfg, x, residual, weight, sum, y, q, q_scale, stream)
PyObject* add_norm(Args a) {
    const auto c = a.description<moe_norm_cfg>(2);
    const auto dt = a.type(c.dtype);
    const int64_t n = static_cast<int64_t>(c.T) * c.d, groups = c.T * static_cast<int64_t>(c.q_group > 0 ? c.d / c.q_group : 1);
    void *x = a.array(3, dt, n), *residual = a.array(4, dt, n), *weight = a.array(5, dt, c.d), *sum = a.array(6, dt, n), *y = a.array(7, dt, n);
    void *q = a.array(8, at::kFloat8_e4m3fn, n), *q_scale = a.array(9, at::kFloat, groups), *stream = a.stream(10);
    auto* f = a.function<decltype(moe_add_norm)>(0);
    return outcome(a, [&] { return f(&c, x, residual, weight, sum, y, q, static_cast<float*>(q_scale), stream); });
}

struct Pages {
    void *k, *v;
    float *k_scales, *v_scales;
    Pages(Args& a, const moe_kv_cfg& c, int at) {
        const int64_t rows = static_cast<int64_t>(c.pages) * c.heads * c.page_size;
        const auto type = a.type(c.cache_dtype);
        k = a.array(at, type, rows * c.head_dim);
        v = a.array(at + 1, type, rows * c.head_dim);
        k_scales = static_cast<float*>(a.array(at + 2, at::kFloat, rows));
        v_scales = static_cast<float*>(a.array(at + 3, at::kFloat, rows));
    }
};

// Tokens: the length of the slots' array.
int64_t length(Args& a, int i) {
    const at::Tensor* t = a.tensor(i);
    if (t == nullptr || t->numel() >= int64_t(1) << 31) a.ok = false;
    return a.ok ? t->numel() : 0;
}

// (function, -, cfg, k, v, slots, k_pages, v_pages, k_scales, v_scales, stream)
PyObject* kv_write(Args a) {
    const auto c = a.description<moe_kv_cfg>(2);
    const int64_t n = length(a, 5);
    int64_t ks, vs;
    void *k = a.rows(3, a.type(c.dtype), n, c.heads, c.head_dim, &ks), *v = a.rows(4, a.type(c.dtype), n, c.heads, c.head_dim, &vs);
    auto* slots = static_cast<const int32_t*>(a.array(5, at::kInt, n));
    const Pages p(a, c, 6);
    void* stream = a.stream(10);
    auto* f = a.function<decltype(moe_kv_write)>(0);
    return outcome(a, [&] { return f(&c, static_cast<int32_t>(n), k, ks, v, vs, slots, p.k, p.v, p.k_scales, p.v_scales, stream); });
}

// (function, -, cfg, k_pages, v_pages, k_scales, v_scales, slots, k, v, stream)
PyObject* kv_read(Args a) {
    const auto c = a.description<moe_kv_cfg>(2);
    const int64_t n = length(a, 7);
    int64_t ks, vs;
    void *k = a.rows(8, a.type(c.dtype), n, c.heads, c.head_dim, &ks), *v = a.rows(9, a.type(c.dtype), n, c.heads, c.head_dim, &vs);
    auto* slots = static_cast<const int32_t*>(a.array(7, at::kInt, n));
    const Pages p(a, c, 3);
    void* stream = a.stream(10);
    auto* f = a.function<decltype(moe_kv_read)>(0);
    return outcome(a, [&] { return f(&c, static_cast<int32_t>(n), p.k, p.v, p.k_scales, p.v_scales, slots, k, ks, v, vs, stream); });
}

// (function, moe_attn_workspace_bytes, cfg, attn, q, k_pages, v_pages, k_scales, v_scales, table, lens, out, lse, ws, stream)
PyObject* attn_decode(Args a) {
    const auto c = a.description<moe_kv_cfg>(2);
    const auto t = a.description<moe_attn_cfg>(3);
    const auto dt = a.type(c.dtype);
    const int64_t heads = static_cast<int64_t>(t.B) * t.q_heads;
    int64_t qs;
    void* q = a.rows(4, dt, t.B, t.q_heads, c.head_dim, &qs);
    const Pages p(a, c, 5);
    auto* table = static_cast<const int32_t*>(a.array(9, at::kInt, static_cast<int64_t>(t.B) * t.table_pages));
    auto* lens = static_cast<const int32_t*>(a.array(10, at::kInt, t.B));
    void *out = a.array(11, dt, heads * c.head_dim), *lse = a.array(12, at::kFloat, heads), *ws = nullptr;
    if (const at::Tensor* w = a.tensor(13)) {
        size_t need = 0;
        if (!a.ok || !w->is_contiguous() || a.function<decltype(moe_attn_workspace_bytes)>(1)(&c, &t, &need) != 0 || w->nbytes() < need) a.ok = false;
        else ws = w->data_ptr();
    }
    void* stream = a.stream(14);
    auto* f = a.function<decltype(moe_attn_decode)>(0);
    return outcome(a, [&] { return f(&c, &t, q, qs, p.k, p.v, p.k_scales, p.v_scales, table, lens, out, static_cast<float*>(lse), ws, stream); });
}

template <PyObject* (*F)(Args), int N>
PyObject* entry(PyObject* self, PyObject* const* at, Py_ssize_t n) { return guarded<F>(self, at, n, N); }

template <PyObject* (*F)(Args), int N>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<F, N>)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<add_norm, 11>("add_norm"), method<kv_write, 11>("kv_write"), method<kv_read, 11>("kv_read"),
                         method<attn_decode, 15>("attn_decode"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__args() { return PyModule_Create(&module_def); }
