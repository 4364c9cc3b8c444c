// The calls of norms and attention from Python, as operators.hpp has them: ordinary ones are
// carried out, any other gives None.
#pragma once

#include "operators.hpp"

namespace operators {

inline PyObject* wrap_all(std::initializer_list<at::Tensor*> tensors) {
    auto out = pybind11::reinterpret_steal<pybind11::object>(PyTuple_New((Py_ssize_t)tensors.size()));
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (at::Tensor* t : tensors) {
        PyObject* o = THPVariable_Wrap(std::move(*t));
        if (!o) return nullptr;
        PyTuple_SET_ITEM(out.ptr(), i++, o);
    }
    return out.release().ptr();
}

inline at::Tensor floats(const at::Tensor& like, at::IntArrayRef shape) {
    return at::empty(shape, like.options().dtype(at::kFloat).requires_grad(false));
}

// norm_kept(call, x, gain, residual, eps, device, stream): (norm, inverse root mean squares)
// or (norm, inverses, h), for the gradient.
inline PyObject* norm_kept(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(7, "norm_kept(call, x, gain, residual, eps, device, stream)")
    typedef int32_t (*Call)(const sllm_matrix*, const sllm_matrix*, const sllm_matrix*, float, const sllm_matrix*, const sllm_matrix*, float*,
                            int32_t, void*);
    const auto call = address<Call>(args[0]);
    const double eps = PyFloat_AsDouble(args[4]);
    const long device = PyLong_AsLong(args[5]);
    void* const stream = PyLong_AsVoidPtr(args[6]);
    if (PyErr_Occurred()) return nullptr;
    const bool has_residual = args[3] != Py_None;
    const at::Tensor *x = tensor(args[1], device), *gain = tensor(args[2], device), *residual = has_residual ? tensor(args[3], device) : nullptr;
    sllm_matrix rows, gain_row, residual_rows, h_rows, y_rows;
    if (!x || !gain || (has_residual && !residual) || !rows_of(*x, &rows) || gain->dim() != 1 || !rows_of(*gain, &gain_row)) Py_RETURN_NONE;
    if (has_residual && (residual->sizes() != x->sizes() || !rows_of(*residual, &residual_rows))) Py_RETURN_NONE;
    at::Tensor h, y = make(*x, x->sizes(), rows.rows, rows.dtype, &y_rows), inverse = floats(*x, {(int64_t)rows.rows});
    if (has_residual) h = make(*x, x->sizes(), rows.rows, rows.dtype, &h_rows);
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        code = call(&rows, has_residual ? &residual_rows : nullptr, &gain_row, (float)eps, has_residual ? &h_rows : nullptr, &y_rows,
                    inverse.data_ptr<float>(), (int32_t)device, stream);
    }
    if (code != SLLM_OK) return PyLong_FromLong(code);
    return has_residual ? wrap_all({&y, &inverse, &h}) : wrap_all({&y, &inverse});
    END_HANDLE_TH_ERRORS
}

// norm_grad(call, workspace, dy, dh, h, gain, inverse, device, stream): (dx, dgain)
inline PyObject* norm_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(9, "norm_grad(call, workspace, dy, dh, h, gain, inverse, device, stream)")
    typedef int32_t (*Call)(const sllm_matrix*, const sllm_matrix*, const sllm_matrix*, const sllm_matrix*, const float*, const sllm_matrix*,
                            const sllm_matrix*, void*, uint64_t, int32_t, void*);
    typedef int32_t (*Workspace)(uint64_t, uint64_t, uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long device = PyLong_AsLong(args[7]);
    void* const stream = PyLong_AsVoidPtr(args[8]);
    if (PyErr_Occurred()) return nullptr;
    const bool has_dh = args[3] != Py_None;
    const at::Tensor *dy = tensor(args[2], device), *dh = has_dh ? tensor(args[3], device) : nullptr, *h = tensor(args[4], device),
                     *gain = tensor(args[5], device), *inverse = tensor(args[6], device);
    sllm_matrix dy_rows, dh_rows, h_rows, gain_row, dx_rows, dgain_row;
    if (!dy || (has_dh && !dh) || !h || !gain || !inverse || !rows_of(*dy, &dy_rows) || (has_dh && !rows_of(*dh, &dh_rows)) ||
        !rows_of(*h, &h_rows) || !rows_of(*gain, &gain_row) || inverse->scalar_type() != at::kFloat || inverse->numel() != (int64_t)h_rows.rows ||
        !inverse->is_contiguous())
        Py_RETURN_NONE;
    at::Tensor dx = make(*h, h->sizes(), h_rows.rows, h_rows.dtype, &dx_rows), dgain = make(*gain, gain->sizes(), 1, gain_row.dtype, &dgain_row), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(h_rows.rows, h_rows.cols, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*h, 1, (int64_t)n);
            code = call(&dy_rows, has_dh ? &dh_rows : nullptr, &h_rows, &gain_row, inverse->data_ptr<float>(), &dx_rows, &dgain_row,
                        n ? ws.data_ptr() : nullptr, n, (int32_t)device, stream);
        }
    }
    if (code != SLLM_OK) return PyLong_FromLong(code);
    return wrap_all({&dx, &dgain});
    END_HANDLE_TH_ERRORS
}

// norm(call, x, gain, residual, eps, mx8, device, stream): the norm, and with a residual
// (norm, h); with mx8 (codes, scales) or (codes, scales, h).
inline PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(8, "norm(call, x, gain, residual, eps, mx8, device, stream)")
    typedef int32_t (*Call)(const sllm_matrix*, const sllm_matrix*, const sllm_matrix*, float, const sllm_matrix*, const sllm_matrix*, float*,
                            int32_t, void*);
    typedef int32_t (*OctetCall)(const sllm_matrix*, const sllm_matrix*, const sllm_matrix*, float, const sllm_matrix*, const sllm_mx*, int32_t,
                                 void*);
    void* const call = PyLong_AsVoidPtr(args[0]);
    const double eps = PyFloat_AsDouble(args[4]);
    const long mx8 = PyLong_AsLong(args[5]), device = PyLong_AsLong(args[6]);
    void* const stream = PyLong_AsVoidPtr(args[7]);
    if (PyErr_Occurred()) return nullptr;
    const bool has_residual = args[3] != Py_None;
    const at::Tensor *x = tensor(args[1], device), *gain = tensor(args[2], device), *residual = has_residual ? tensor(args[3], device) : nullptr;
    sllm_matrix rows, gain_row, residual_rows, h_rows, y_rows;
    if (!x || !gain || (has_residual && !residual) || !rows_of(*x, &rows) || gain->dim() != 1 || !rows_of(*gain, &gain_row)) Py_RETURN_NONE;
    if (has_residual && (residual->sizes() != x->sizes() || !rows_of(*residual, &residual_rows))) Py_RETURN_NONE;
    at::Tensor h, y, scales;
    if (has_residual) h = make(*x, x->sizes(), rows.rows, rows.dtype, &h_rows);
    sllm_mx q;
    if (mx8) {
        const int64_t blocks = ((int64_t)rows.cols + 31) / 32;
        y = bytes(*x, (int64_t)rows.rows, blocks * 32);
        scales = bytes(*x, (int64_t)rows.rows, (blocks + 15) / 16 * 16);
        q = sllm_mx{y.data_ptr(), scales.data_ptr(), rows.rows, rows.cols};
    } else {
        y = make(*x, x->sizes(), rows.rows, rows.dtype, &y_rows);
    }
    const sllm_matrix *r = has_residual ? &residual_rows : nullptr, *to = has_residual ? &h_rows : nullptr;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        code = mx8 ? reinterpret_cast<OctetCall>(call)(&rows, r, &gain_row, (float)eps, to, &q, (int32_t)device, stream)
                   : reinterpret_cast<Call>(call)(&rows, r, &gain_row, (float)eps, to, &y_rows, nullptr, (int32_t)device, stream);
    }
    if (code != SLLM_OK) return PyLong_FromLong(code);
    if (mx8) return has_residual ? wrap_all({&y, &scales, &h}) : wrap_all({&y, &scales});
    if (has_residual) return wrap_all({&y, &h});
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

// product_octet(call, workspace, x's codes, scales, cols, w's codes, scales, cols, dtype,
// device, stream): x @ w.T, x in MX FP8 and w in MX FP4.
inline PyObject* product_octet(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(11, "product_octet(call, workspace, codes, scales, cols, codes, scales, cols, dtype, device, stream)")
    typedef int32_t (*Call)(const sllm_mx*, const sllm_mx*, const sllm_matrix*, void*, uint64_t, int32_t, void*);
    typedef int32_t (*Workspace)(const sllm_mx*, const sllm_mx*, uint32_t, uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long type = PyLong_AsLong(args[8]), device = PyLong_AsLong(args[9]);
    void* const stream = PyLong_AsVoidPtr(args[10]);
    if (PyErr_Occurred()) return nullptr;
    sllm_mx x, w;
    const at::Tensor* codes = mx_of(args[2], args[3], args[4], device, &x, 32);
    if (!codes || !mx_of(args[5], args[6], args[7], device, &w) || !x.rows || !w.rows || x.cols != w.cols) Py_RETURN_NONE;
    sllm_matrix out_rows;
    at::Tensor out = make(*codes, {(int64_t)x.rows, (int64_t)w.rows}, x.rows, (uint32_t)type, &out_rows), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(&x, &w, (uint32_t)type, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*codes, 1, (int64_t)n);
            code = call(&x, &w, &out_rows, n ? ws.data_ptr() : nullptr, n, (int32_t)device, stream);
        }
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

// (tokens, heads, elements) by their strides.
inline bool heads_of(const at::Tensor* t, sllm_heads* out) {
    uint32_t code;
    if (!t || !dtype_code(t->scalar_type(), &code) || t->dim() != 3 || !t->numel()) return false;
    const int64_t tokens = t->size(0), heads = t->size(1), dim = t->size(2);
    if ((dim > 1 && t->stride(2) != 1) || t->stride(0) < 0 || t->stride(1) < 0) return false;
    *out = sllm_heads{t->data_ptr(), (uint64_t)tokens, (uint64_t)heads, (uint64_t)dim, (uint64_t)(tokens > 1 ? t->stride(0) : heads * dim),
                      (uint64_t)(heads > 1 ? t->stride(1) : dim), code, 0};
    return true;
}

// A list of numbers, if there is one.
inline bool list_of(PyObject* o, int64_t device, sllm_ids* ids, const sllm_ids** p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = tensor(o, device);
    if (!t || t->dim() != 1 || !ids_of(*t, ids)) return false;
    *p = ids;
    return true;
}

inline at::Tensor like_heads(const at::Tensor& q, const sllm_heads& from, sllm_heads* to) {
    at::Tensor t = at::empty(q.sizes(), q.options().requires_grad(false));
    *to = sllm_heads{t.data_ptr(), from.tokens, from.heads, from.dim, from.heads * from.dim, from.dim, from.dtype, 0};
    return t;
}

// attention(call, q, k, v, offsets, window, sinks, scale, device, stream, keep): the output,
// or with `keep` (output, lse), for the gradient.
inline PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(11, "attention(call, q, k, v, offsets, window, sinks, scale, device, stream, keep)")
    typedef int32_t (*Call)(const sllm_heads*, const sllm_heads*, const sllm_heads*, const sllm_ids*, uint64_t, uint64_t, float,
                            const sllm_heads*, float*, int32_t, void*);
    const auto call = address<Call>(args[0]);
    const long long window = PyLong_AsLongLong(args[5]), sinks = PyLong_AsLongLong(args[6]);
    const double scale = PyFloat_AsDouble(args[7]);
    const long device = PyLong_AsLong(args[8]);
    void* const stream = PyLong_AsVoidPtr(args[9]);
    const long keep = PyLong_AsLong(args[10]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* q = tensor(args[1], device);
    sllm_heads q_rows, k_rows, v_rows, out_rows;
    sllm_ids ids;
    const sllm_ids* offsets;
    if (!heads_of(q, &q_rows) || !heads_of(tensor(args[2], device), &k_rows) || !heads_of(tensor(args[3], device), &v_rows) ||
        !list_of(args[4], device, &ids, &offsets) || window < 0 || sinks < 0)
        Py_RETURN_NONE;
    at::Tensor out = like_heads(*q, q_rows, &out_rows), lse;
    if (keep) lse = floats(*q, {q->size(0), q->size(1)});
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        code = call(&q_rows, &k_rows, &v_rows, offsets, (uint64_t)window, (uint64_t)sinks, (float)scale, &out_rows,
                    keep ? lse.data_ptr<float>() : nullptr, (int32_t)device, stream);
    }
    if (code == SLLM_OK && keep) return wrap_all({&out, &lse});
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

// attention_grad(call, workspace, dout, q, k, v, out, lse, offsets, window, sinks, scale,
// device, stream): (dq, dk, dv)
inline PyObject* attention_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(14, "attention_grad(call, workspace, dout, q, k, v, out, lse, offsets, window, sinks, scale, device, stream)")
    typedef int32_t (*Call)(const sllm_heads*, const sllm_heads*, const sllm_heads*, const sllm_heads*, const sllm_heads*, const float*,
                            const sllm_ids*, uint64_t, uint64_t, float, const sllm_heads*, const sllm_heads*, const sllm_heads*, void*, uint64_t,
                            int32_t, void*);
    typedef int32_t (*Workspace)(const sllm_heads*, const sllm_heads*, const sllm_ids*, uint64_t, uint64_t, uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long long window = PyLong_AsLongLong(args[9]), sinks = PyLong_AsLongLong(args[10]);
    const double scale = PyFloat_AsDouble(args[11]);
    const long device = PyLong_AsLong(args[12]);
    void* const stream = PyLong_AsVoidPtr(args[13]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *q = tensor(args[3], device), *k = tensor(args[4], device), *v = tensor(args[5], device), *lse = tensor(args[7], device);
    sllm_heads dout, q_rows, k_rows, v_rows, out, dq_rows, dk_rows, dv_rows;
    sllm_ids ids;
    const sllm_ids* offsets;
    if (!heads_of(tensor(args[2], device), &dout) || !heads_of(q, &q_rows) || !heads_of(k, &k_rows) || !heads_of(v, &v_rows) ||
        !heads_of(tensor(args[6], device), &out) || !lse || lse->scalar_type() != at::kFloat || !lse->is_contiguous() ||
        lse->numel() != q->size(0) * q->size(1) || !list_of(args[8], device, &ids, &offsets) || window < 0 || sinks < 0)
        Py_RETURN_NONE;
    at::Tensor dq = like_heads(*q, q_rows, &dq_rows), dk = like_heads(*k, k_rows, &dk_rows), dv = like_heads(*v, v_rows, &dv_rows), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(&q_rows, &k_rows, offsets, (uint64_t)window, (uint64_t)sinks, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*q, 1, (int64_t)n);
            code = call(&dout, &q_rows, &k_rows, &v_rows, &out, lse->data_ptr<float>(), offsets, (uint64_t)window, (uint64_t)sinks, (float)scale,
                        &dq_rows, &dk_rows, &dv_rows, n ? ws.data_ptr() : nullptr, n, (int32_t)device, stream);
        }
    }
    if (code != SLLM_OK) return PyLong_FromLong(code);
    return wrap_all({&dq, &dk, &dv});
    END_HANDLE_TH_ERRORS
}

// attention_cached(call, workspace, q, k, v, cached k, cached v, window, sinks, lengths,
// offsets, scale, device, stream)
inline PyObject* attention_cached(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    SLLM_PY_ARGS(14, "attention_cached(call, workspace, q, k, v, k, v, window, sinks, lengths, offsets, scale, device, stream)")
    typedef int32_t (*Call)(const sllm_heads*, const sllm_heads*, const sllm_heads*, const sllm_kv_cache*, const sllm_ids*, const sllm_ids*, float,
                            const sllm_heads*, void*, uint64_t, int32_t, void*);
    typedef int32_t (*Workspace)(const sllm_heads*, const sllm_heads*, const sllm_heads*, const sllm_kv_cache*, const sllm_ids*, const sllm_ids*,
                                 uint64_t*);
    const auto call = address<Call>(args[0]);
    const auto workspace = address<Workspace>(args[1]);
    const long long window = PyLong_AsLongLong(args[7]), sinks = PyLong_AsLongLong(args[8]);
    const double scale = PyFloat_AsDouble(args[11]);
    const long device = PyLong_AsLong(args[12]);
    void* const stream = PyLong_AsVoidPtr(args[13]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *q = tensor(args[2], device), *ck = tensor(args[5], device), *cv = tensor(args[6], device);
    sllm_heads q_rows, k_rows, v_rows, out_rows;
    sllm_ids length_ids, offset_ids;
    const sllm_ids *lengths, *offsets;
    if (!heads_of(q, &q_rows) || !heads_of(tensor(args[3], device), &k_rows) || !heads_of(tensor(args[4], device), &v_rows) || !ck || !cv ||
        !list_of(args[9], device, &length_ids, &lengths) || !lengths || !list_of(args[10], device, &offset_ids, &offsets) || window < 1 || sinks < 0)
        Py_RETURN_NONE;
    uint32_t type;
    if (ck->dim() != 4 || ck->sizes() != cv->sizes() || ck->scalar_type() != cv->scalar_type() || !dtype_code(ck->scalar_type(), &type) ||
        !ck->is_contiguous() || !cv->is_contiguous() || ck->size(2) != window + sinks)
        Py_RETURN_NONE;
    const sllm_kv_cache cache{ck->data_ptr(), cv->data_ptr(), (uint64_t)ck->size(0), (uint64_t)ck->size(1), (uint64_t)ck->size(3),
                              (uint64_t)window, (uint64_t)sinks, type, 0};
    at::Tensor out = like_heads(*q, q_rows, &out_rows), ws;
    int32_t code;
    {
        pybind11::gil_scoped_release no_gil;
        uint64_t n = 0;
        code = workspace(&q_rows, &k_rows, &v_rows, &cache, lengths, offsets, &n);
        if (code == SLLM_OK) {
            if (n) ws = bytes(*q, 1, (int64_t)n);
            code = call(&q_rows, &k_rows, &v_rows, &cache, lengths, offsets, (float)scale, &out_rows, n ? ws.data_ptr() : nullptr, n,
                        (int32_t)device, stream);
        }
    }
    return result(code, std::move(out));
    END_HANDLE_TH_ERRORS
}

#undef SLLM_PY_ARGS

}  // namespace operators
