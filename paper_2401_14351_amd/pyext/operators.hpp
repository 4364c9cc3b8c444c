// The operators' calls from Python: operands described, the result and its
// workspace allocated and the C entry point called in one go.
//
// A small operator's kernel takes 3 to 9 us, and its call from Python took longer:
// 8.5 us, of which 4 are the entry point's (its checks and the launch) and the rest
// the interpreter's.  These functions take the ordinary call, tensors on a GPU whose
// rows need no second look, and return None for any other: Python then carries it
// out, or says what is wrong with it.  A failed call's code is returned as a number.
//
// Entry points come as addresses, so this extension needs nothing of libsllm.so.
#pragma once

#include <Python.h>

#include <ATen/Functions.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "sllm.h"

namespace operators {

inline bool dtype_code(at::ScalarType type, uint32_t* code) {
    *code = type == at::kFloat ? SLLM_DTYPE_F32 : type == at::kHalf ? SLLM_DTYPE_F16 : SLLM_DTYPE_BF16;
    return type == at::kFloat || type == at::kHalf || type == at::kBFloat16;
}

constexpr at::ScalarType kTypes[] = {at::kFloat, at::kHalf, at::kBFloat16};  // by SLLM_DTYPE_*

// A tensor argument, or null where it is not a plain tensor on `device`.
inline const at::Tensor* tensor(PyObject* o, int64_t device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.get_device() == device && !t.is_neg() ? &t : nullptr;
}

// The rows of t, its last dimension's runs of elements.
inline bool rows_of(const at::Tensor& t, sllm_matrix* m) {
    uint32_t code;
    const int64_t dim = t.dim();
    if (!dtype_code(t.scalar_type(), &code) || dim < 1) return false;
    const int64_t cols = t.size(dim - 1);
    const int64_t rows = dim == 1 ? 1 : dim == 2 ? t.size(0) : cols ? t.numel() / cols : 0;
    if (!rows || !cols || (dim > 2 && !t.is_contiguous()) || (cols > 1 && t.stride(dim - 1) != 1)) return false;
    const int64_t stride = dim == 2 && rows > 1 ? t.stride(0) : cols;
    if (stride < 0) return false;
    *m = sllm_matrix{t.data_ptr(), (uint64_t)rows, (uint64_t)cols, (uint64_t)stride, code, 0};
    return true;
}

inline bool ids_of(const at::Tensor& t, sllm_ids* ids) {
    const bool wide = t.scalar_type() == at::kLong;
    if ((!wide && t.scalar_type() != at::kInt) || !t.is_contiguous() || !t.numel()) return false;
    *ids = sllm_ids{t.data_ptr(), (uint64_t)t.numel(), wide ? 64u : 32u, 0};
    return true;
}

// A matrix in MX FP4, or with blocks of 32 bytes FP8, from its tensors; null codes where they are not what it is made of.
// Gives the codes' tensor, which tells where results are allocated.
inline const at::Tensor* mx_of(PyObject* codes, PyObject* scales, PyObject* cols, int64_t device, sllm_mx* q, int64_t block = 16) {
    const long long n = PyLong_AsLongLong(cols);
    if (n < 0) {
        PyErr_Clear();
        return nullptr;
    }
    const int64_t blocks = (n + 31) / 32;
    const at::Tensor *c = tensor(codes, device), *s = tensor(scales, device);
    const auto fits = [](const at::Tensor* t, int64_t pitch) {
        return t && t->scalar_type() == at::kByte && t->dim() == 2 && t->size(1) == pitch && t->is_contiguous();
    };
    if (!fits(c, blocks * block) || !fits(s, (blocks + 15) / 16 * 16) || c->size(0) != s->size(0)) return nullptr;
    *q = sllm_mx{c->data_ptr(), s->data_ptr(), (uint64_t)c->size(0), (uint64_t)n};
    return c;
}

// A new tensor beside `like`, and its rows.
inline at::Tensor make(const at::Tensor& like, at::IntArrayRef shape, uint64_t rows, uint32_t code, sllm_matrix* m) {
    at::Tensor t = at::empty(shape, like.options().dtype(kTypes[code]).requires_grad(false));
    const uint64_t cols = (uint64_t)shape.back();
    *m = sllm_matrix{t.data_ptr(), rows, cols, cols, code, 0};
    return t;
}

inline at::Tensor bytes(const at::Tensor& like, int64_t rows, int64_t n) {
    return at::empty({rows, n}, like.options().dtype(at::kByte).requires_grad(false));
}

inline PyObject* result(int32_t code, at::Tensor&& t) {
    return code == SLLM_OK ? THPVariable_Wrap(std::move(t)) : PyLong_FromLong(code);
}

template <typename T>
T address(PyObject* o) {
    return reinterpret_cast<T>(PyLong_AsVoidPtr(o));
}

#define SLLM_PY_ARGS(n, what)                    \
    if (nargs != n) {                            \
        PyErr_SetString(PyExc_TypeError, what);  \
        return nullptr;                          \
    }

// product(call, workspace, x, codes, scales, cols, dtype, grad, device, stream): x @ w.T,
// or with `grad` x @ w.  dtype as SLLM_DTYPE_*, or -1 for x's.
inline PyObject* product(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(10, "product(call, workspace, x, codes, scales, cols, dtype, grad, device, stream)")
    typedef int32_t (*Call)(const sllm_matrix*, const sllm_mx*, const sllm_matrix*, void*, uint64_t, int32_t, void*);
    typedef int32_t (*Workspace)(const sllm_matrix*, const sllm_mx*, uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long type = PyLong_AsLong(args[6]), grad = PyLong_AsLong(args[7]), device = PyLong_AsLong(args[8]);
    void* const stream = PyLong_AsVoidPtr(args[9]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* x = tensor(args[2], device);
    sllm_matrix rows, out_rows;
    sllm_mx w;
    if (!x || !rows_of(*x, &rows) || !mx_of(args[3], args[4], args[5], device, &w)) Py_RETURN_NONE;
    const uint64_t cols = grad ? w.cols : w.rows;
    if (!cols || rows.cols != (grad ? w.rows : w.cols)) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 4> shape(x->sizes().begin(), x->sizes().end());
    shape.back() = (int64_t)cols;
    at::Tensor out = make(*x, shape, rows.rows, type < 0 ? rows.dtype : (uint32_t)type, &out_rows), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(&rows, &w, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*x, 1, (int64_t)n);
            code = call(&rows, &w, &out_rows, n ? ws.data_ptr() : nullptr, n, (int32_t)device, stream);
        }
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

// product_mx(call, workspace, x's codes, scales, cols, w's codes, scales, cols, dtype, device,
// stream): the same with x in MX FP4.
inline PyObject* product_mx(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(11, "product_mx(call, workspace, codes, scales, cols, codes, scales, cols, dtype, device, stream)")
    typedef int32_t (*Call)(const sllm_mx*, const sllm_mx*, const sllm_matrix*, void*, uint64_t, int32_t, void*);
    typedef int32_t (*Workspace)(const sllm_mx*, const sllm_mx*, uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long type = PyLong_AsLong(args[8]), device = PyLong_AsLong(args[9]);
    void* const stream = PyLong_AsVoidPtr(args[10]);
    if (PyErr_Occurred()) return nullptr;
    sllm_mx x, w;
    const at::Tensor* codes = mx_of(args[2], args[3], args[4], device, &x);
    if (!codes || !mx_of(args[5], args[6], args[7], device, &w) || !x.rows || !w.rows || x.cols != w.cols) Py_RETURN_NONE;
    sllm_matrix out_rows;
    at::Tensor out = make(*codes, {(int64_t)x.rows, (int64_t)w.rows}, x.rows, (uint32_t)type, &out_rows), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(&x, &w, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*codes, 1, (int64_t)n);
            code = call(&x, &w, &out_rows, n ? ws.data_ptr() : nullptr, n, (int32_t)device, stream);
        }
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

// quantize(call, x, device, stream) -> (codes, scales)
inline PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(4, "quantize(call, x, device, stream)")
    typedef int32_t (*Call)(const sllm_matrix*, const sllm_mx*, int32_t, void*);
    const auto call = address<Call>(args[0]);
    const long device = PyLong_AsLong(args[2]);
    void* const stream = PyLong_AsVoidPtr(args[3]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* x = tensor(args[1], device);
    sllm_matrix rows;
    if (!x || !rows_of(*x, &rows)) Py_RETURN_NONE;
    const int64_t blocks = ((int64_t)rows.cols + 31) / 32;
    at::Tensor codes = bytes(*x, (int64_t)rows.rows, blocks * 16), scales = bytes(*x, (int64_t)rows.rows, (blocks + 15) / 16 * 16);
    const sllm_mx q{codes.data_ptr(), scales.data_ptr(), rows.rows, rows.cols};
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        code = call(&rows, &q, (int32_t)device, stream);
    }
    if (code != SLLM_OK) return PyLong_FromLong(code);
    auto c = pybind11::reinterpret_steal<pybind11::object>(THPVariable_Wrap(std::move(codes)));
    auto s = pybind11::reinterpret_steal<pybind11::object>(THPVariable_Wrap(std::move(scales)));
    return c && s ? PyTuple_Pack(2, c.ptr(), s.ptr()) : nullptr;
    END_HANDLE_TH_ERRORS
}

// dequantize(call, codes, scales, cols, dtype, device, stream)
inline PyObject* dequantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(7, "dequantize(call, codes, scales, cols, dtype, device, stream)")
    typedef int32_t (*Call)(const sllm_mx*, const sllm_matrix*, int32_t, void*);
    const auto call = address<Call>(args[0]);
    const long type = PyLong_AsLong(args[4]), device = PyLong_AsLong(args[5]);
    void* const stream = PyLong_AsVoidPtr(args[6]);
    if (PyErr_Occurred()) return nullptr;
    sllm_mx q;
    const at::Tensor* codes = mx_of(args[1], args[2], args[3], device, &q);
    if (!codes || !q.rows || !q.cols) Py_RETURN_NONE;
    sllm_matrix out_rows;
    at::Tensor out = make(*codes, {(int64_t)q.rows, (int64_t)q.cols}, q.rows, (uint32_t)type, &out_rows);
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        code = call(&q, &out_rows, (int32_t)device, stream);
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

// lookup(call, table, scales, cols, tokens, scale, dtype, device, stream): table a tensor
// and scales None, or the codes of one in MX FP4.
inline PyObject* lookup(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(9, "lookup(call, table, scales, cols, tokens, scale, dtype, device, stream)")
    typedef int32_t (*Call)(const void*, const sllm_ids*, float, const sllm_matrix*, int32_t, void*);
    const bool mx = args[2] != Py_None;
    const double scale = PyFloat_AsDouble(args[5]);
    const long type = PyLong_AsLong(args[6]), device = PyLong_AsLong(args[7]);
    void* const stream = PyLong_AsVoidPtr(args[8]);
    const auto call = address<Call>(args[0]);
    if (PyErr_Occurred()) return nullptr;
    sllm_matrix rows, out_rows;
    sllm_mx q;
    sllm_ids ids;
    const at::Tensor *like = mx ? mx_of(args[1], args[2], args[3], device, &q) : tensor(args[1], device), *tokens = tensor(args[4], device);
    if (!like || !tokens || !ids_of(*tokens, &ids)) Py_RETURN_NONE;
    if (!mx && (like->dim() != 2 || !rows_of(*like, &rows))) Py_RETURN_NONE;
    const void* const table = mx ? static_cast<const void*>(&q) : &rows;
    const uint64_t cols = mx ? q.cols : rows.cols;
    if (!cols) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 4> shape(tokens->sizes().begin(), tokens->sizes().end());
    shape.push_back((int64_t)cols);
    at::Tensor out = make(*like, shape, ids.n, type < 0 ? rows.dtype : (uint32_t)type, &out_rows);
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        code = call(table, &ids, (float)scale, &out_rows, (int32_t)device, stream);
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

// lookup_grad(call, workspace, dy, tokens, vocab, scale, dtype, device, stream)
inline PyObject* lookup_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(9, "lookup_grad(call, workspace, dy, tokens, vocab, scale, dtype, device, stream)")
    typedef int32_t (*Call)(const sllm_matrix*, const sllm_ids*, float, uint32_t, const sllm_matrix*, void*, uint64_t, int32_t, void*);
    typedef int32_t (*Workspace)(uint64_t, const sllm_matrix*, uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long long vocab = PyLong_AsLongLong(args[4]);
    const double scale = PyFloat_AsDouble(args[5]);
    const long type = PyLong_AsLong(args[6]), device = PyLong_AsLong(args[7]);
    void* const stream = PyLong_AsVoidPtr(args[8]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *dy = tensor(args[2], device), *tokens = tensor(args[3], device);
    sllm_matrix rows, out_rows;
    sllm_ids ids;
    if (!dy || !tokens || vocab < 1 || !rows_of(*dy, &rows) || !ids_of(*tokens, &ids) || rows.rows != ids.n) Py_RETURN_NONE;
    at::Tensor out = make(*dy, {(int64_t)vocab, (int64_t)rows.cols}, (uint64_t)vocab, type < 0 ? rows.dtype : (uint32_t)type, &out_rows), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(ids.n, &out_rows, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*dy, 1, (int64_t)n);
            code = call(&rows, &ids, (float)scale, 0, &out_rows, n ? ws.data_ptr() : nullptr, n, (int32_t)device, stream);
        }
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

}  // namespace operators
