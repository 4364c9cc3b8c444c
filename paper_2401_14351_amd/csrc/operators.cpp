// Entry points of the operators on loaded weights: argument checks, then the
// launchers of mx.hip and embedding.hip.
#include "operators.hpp"

#include "common.hpp"
#include "hip_util.hpp"

namespace sllm {

namespace {

// A run of bytes an operator reads or writes.
struct Span {
    const char* name;
    const uint8_t* p;
    uint64_t bytes;
};

int32_t check_extent(const char* name, uint64_t rows, uint64_t cols) {
    if (rows > SLLM_MAX_EXTENT || cols > SLLM_MAX_EXTENT)
        return fail(SLLM_E_RANGE, "%s: %llu x %llu is larger than %llu rows or columns", name, (unsigned long long)rows,
                    (unsigned long long)cols, (unsigned long long)SLLM_MAX_EXTENT);
    return SLLM_OK;
}

int32_t check_pointer(const Span& s, uint64_t alignment) {
    if (!s.bytes) return SLLM_OK;
    if (!s.p) return fail(SLLM_E_INVAL, "%s: NULL pointer", s.name);
    if (reinterpret_cast<uintptr_t>(s.p) % alignment)
        return fail(SLLM_E_INVAL, "%s must be %llu-byte aligned", s.name, (unsigned long long)alignment);
    return SLLM_OK;
}

uint64_t itemsize(uint32_t dtype) { return dtype == SLLM_DTYPE_F32 ? 4 : 2; }

int32_t matrix_span(const char* name, const sllm_matrix* m, Span* out) {
    if (!m) return fail(SLLM_E_INVAL, "%s: NULL", name);
    if (m->dtype != SLLM_DTYPE_F32 && m->dtype != SLLM_DTYPE_F16 && m->dtype != SLLM_DTYPE_BF16)
        return fail(SLLM_E_INVAL, "%s: dtype %u is not f32, f16 or bf16", name, m->dtype);
    if (m->reserved) return fail(SLLM_E_INVAL, "%s: reserved must be 0", name);
    SLLM_TRY(check_extent(name, m->rows, m->cols));
    const uint64_t size = itemsize(m->dtype);
    uint64_t last = 0;
    if (m->rows > 1) {
        if (m->stride < m->cols)
            return fail(SLLM_E_INVAL, "%s: rows of %llu columns overlap at a stride of %llu", name,
                        (unsigned long long)m->cols, (unsigned long long)m->stride);
        if (!mul_ok(m->rows - 1, m->stride, &last) || !add_ok(last, m->cols, &last) || !mul_ok(last, size, &last))
            return fail(SLLM_E_RANGE, "%s: size overflows", name);
    } else {
        last = m->cols * size;
    }
    *out = Span{name, static_cast<const uint8_t*>(m->data), m->rows && m->cols ? last : 0};
    return check_pointer(*out, size);
}

int32_t mx_spans(const char* codes, const char* scales, const sllm_mx* m, Span* out) {
    if (!m) return fail(SLLM_E_INVAL, "%s: NULL", codes);
    SLLM_TRY(check_extent(codes, m->rows, m->cols));
    out[0] = Span{codes, static_cast<const uint8_t*>(m->codes), m->rows * mx_code_pitch(m->cols)};
    out[1] = Span{scales, static_cast<const uint8_t*>(m->scales), m->rows * mx_scale_pitch(m->cols)};
    SLLM_TRY(check_pointer(out[0], 16));
    return check_pointer(out[1], 16);
}

int32_t ids_span(const sllm_ids* ids, Span* out) {
    if (!ids) return fail(SLLM_E_INVAL, "ids: NULL");
    if (ids->bits != 32 && ids->bits != 64) return fail(SLLM_E_INVAL, "ids: %u bits, not 32 or 64", ids->bits);
    if (ids->reserved) return fail(SLLM_E_INVAL, "ids: reserved must be 0");
    SLLM_TRY(check_extent("ids", ids->n, 0));
    *out = Span{"ids", static_cast<const uint8_t*>(ids->data), ids->n * (ids->bits / 8)};
    return check_pointer(*out, ids->bits / 8);
}

// The spans are device memory, and the first n_out, which are written, overlap
// no other.
int32_t check_spans(const Span* s, int n, int n_out, int32_t device) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n_out; ++j)
            if (i != j && s[i].bytes && s[j].bytes && s[i].p < s[j].p + s[j].bytes && s[j].p < s[i].p + s[i].bytes)
                return fail(SLLM_E_INVAL, "%s and %s overlap", s[i].name, s[j].name);
    for (int i = 0; i < n; ++i) SLLM_TRY(check_device_range(s[i].p, s[i].bytes, device, s[i].name));
    return SLLM_OK;
}

int32_t workspace_span(void* workspace, uint64_t bytes, uint64_t need, Span* out) {
    if (bytes < need)
        return fail(SLLM_E_RANGE, "workspace of %llu bytes, %llu needed", (unsigned long long)bytes,
                    (unsigned long long)need);
    *out = Span{"workspace", static_cast<const uint8_t*>(workspace), need};
    return check_pointer(*out, 16);
}

Operand operand(const sllm_matrix& m) { return Operand{m.data, m.stride, m.dtype, nullptr, nullptr}; }

Operand operand(const sllm_mx& m) {
    return Operand{nullptr, 0, 0, static_cast<const uint8_t*>(m.codes), static_cast<const uint8_t*>(m.scales)};
}

// What a product is of, from its operands: x is a matrix or in MX FP4.
struct LinearArgs {
    LinearLaunch a;
    Span x[2], w[2];
    int n_x = 0;
    uint64_t out_cols = 0;
};

int32_t linear_args(const sllm_matrix* x, const sllm_mx* x_mx, const sllm_mx* w, bool grad, LinearArgs* out) {
    uint64_t rows, cols;
    if (x_mx || !x) {
        SLLM_TRY(mx_spans("x codes", "x scales", x_mx, out->x));
        out->n_x = 2;
        rows = x_mx->rows, cols = x_mx->cols;
        out->a.x = operand(*x_mx);
    } else {
        SLLM_TRY(matrix_span(grad ? "dy" : "x", x, out->x));
        out->n_x = 1;
        rows = x->rows, cols = x->cols;
        out->a.x = operand(*x);
    }
    SLLM_TRY(mx_spans("w codes", "w scales", w, out->w));
    if (cols != (grad ? w->rows : w->cols))
        return fail(SLLM_E_INVAL, "%s has %llu columns, the weight %llu %s", grad ? "dy" : "x", (unsigned long long)cols,
                    (unsigned long long)(grad ? w->rows : w->cols), grad ? "rows" : "columns");
    out->a.m = rows, out->a.n = w->rows, out->a.k = w->cols;
    out->a.w_codes = static_cast<const uint8_t*>(w->codes);
    out->a.w_scales = static_cast<const uint8_t*>(w->scales);
    out->a.grad = grad;
    out->out_cols = grad ? w->cols : w->rows;
    return SLLM_OK;
}

int32_t linear(const sllm_matrix* x, const sllm_mx* x_mx, const sllm_mx* w, const sllm_matrix* out, bool grad,
               void* workspace, uint64_t workspace_bytes, int32_t device, void* stream) {
    LinearArgs l;
    SLLM_TRY(linear_args(x, x_mx, w, grad, &l));
    Span s[6];
    int n = 0;
    SLLM_TRY(matrix_span(grad ? "dx" : "out", out, &s[n++]));
    if (out->rows != l.a.m || out->cols != l.out_cols)
        return fail(SLLM_E_INVAL, "%s is %llu x %llu, not %llu x %llu", grad ? "dx" : "out",
                    (unsigned long long)out->rows, (unsigned long long)out->cols, (unsigned long long)l.a.m,
                    (unsigned long long)l.out_cols);
    l.a.out = out->data;
    l.a.out_stride = out->stride;
    l.a.out_dtype = out->dtype;
    SLLM_TRY(workspace_span(workspace, workspace_bytes, linear_workspace(l.a), &s[n++]));
    for (int i = 0; i < l.n_x; ++i) s[n++] = l.x[i];
    s[n++] = l.w[0];
    s[n++] = l.w[1];
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, n, 2, device));
    if (!l.a.m || !l.out_cols) return SLLM_OK;
    return launch_linear(l.a, workspace, static_cast<hipStream_t>(stream));
}

int32_t linear_bytes(const sllm_matrix* x, const sllm_mx* x_mx, const sllm_mx* w, bool grad, uint64_t* bytes) {
    if (!bytes) return fail(SLLM_E_INVAL, "bytes: NULL");
    LinearArgs l;
    SLLM_TRY(linear_args(x, x_mx, w, grad, &l));
    *bytes = linear_workspace(l.a);
    return SLLM_OK;
}

int32_t embedding(const sllm_matrix* table, const sllm_mx* table_mx, const sllm_ids* ids, float scale,
                  const sllm_matrix* out, int32_t device, void* stream) {
    EmbeddingLaunch a;
    Span s[4];
    int n = 0;
    SLLM_TRY(matrix_span("out", out, &s[n++]));
    if (table_mx || !table) {
        SLLM_TRY(mx_spans("table codes", "table scales", table_mx, &s[n]));
        n += 2;
        a.table = operand(*table_mx);
        a.vocab = table_mx->rows, a.dim = table_mx->cols;
    } else {
        SLLM_TRY(matrix_span("table", table, &s[n++]));
        a.table = operand(*table);
        a.vocab = table->rows, a.dim = table->cols;
    }
    SLLM_TRY(ids_span(ids, &s[n++]));
    if (out->rows != ids->n || out->cols != a.dim)
        return fail(SLLM_E_INVAL, "out is %llu x %llu, not %llu x %llu", (unsigned long long)out->rows,
                    (unsigned long long)out->cols, (unsigned long long)ids->n, (unsigned long long)a.dim);
    a.ids = ids->data, a.ids64 = ids->bits == 64, a.n = ids->n;
    a.scale = scale;
    a.out = out->data, a.out_stride = out->stride, a.out_dtype = out->dtype;
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, n, 1, device));
    if (!a.n || !a.dim) return SLLM_OK;
    return launch_embedding(a, static_cast<hipStream_t>(stream));
}

}  // namespace

}  // namespace sllm

using namespace sllm;

extern "C" int32_t sllm_mx_sizes(uint64_t rows, uint64_t cols, uint64_t* codes_bytes, uint64_t* scales_bytes) try {
    clear_error();
    if (!codes_bytes || !scales_bytes) return fail(SLLM_E_INVAL, "codes_bytes and scales_bytes must be non-NULL");
    SLLM_TRY(check_extent("matrix", rows, cols));
    *codes_bytes = rows * mx_code_pitch(cols);
    *scales_bytes = rows * mx_scale_pitch(cols);
    return SLLM_OK;
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_quantize(const sllm_matrix* src, const sllm_mx* dst, int32_t device, void* stream) try {
    clear_error();
    Span s[3];
    SLLM_TRY(mx_spans("codes", "scales", dst, s));
    SLLM_TRY(matrix_span("source", src, &s[2]));
    if (src->rows != dst->rows || src->cols != dst->cols)
        return fail(SLLM_E_INVAL, "source and destination differ in shape");
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, 3, 2, device));
    if (!src->rows || !src->cols) return SLLM_OK;
    return launch_quantize(*src, *dst, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_dequantize(const sllm_mx* src, const sllm_matrix* dst, int32_t device, void* stream) try {
    clear_error();
    Span s[3];
    SLLM_TRY(matrix_span("destination", dst, &s[0]));
    SLLM_TRY(mx_spans("codes", "scales", src, &s[1]));
    if (src->rows != dst->rows || src->cols != dst->cols)
        return fail(SLLM_E_INVAL, "source and destination differ in shape");
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, 3, 1, device));
    if (!src->rows || !src->cols) return SLLM_OK;
    EmbeddingLaunch a;
    a.table = operand(*src);
    a.vocab = a.n = src->rows, a.dim = src->cols;
    a.out = dst->data, a.out_stride = dst->stride, a.out_dtype = dst->dtype;
    return launch_embedding(a, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_linear(const sllm_matrix* x, const sllm_mx* w, const sllm_matrix* out, void* workspace,
                                  uint64_t workspace_bytes, int32_t device, void* stream) try {
    clear_error();
    if (!x) return fail(SLLM_E_INVAL, "x: NULL");
    return linear(x, nullptr, w, out, false, workspace, workspace_bytes, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_linear_mx(const sllm_mx* x, const sllm_mx* w, const sllm_matrix* out, void* workspace,
                                     uint64_t workspace_bytes, int32_t device, void* stream) try {
    clear_error();
    return linear(nullptr, x, w, out, false, workspace, workspace_bytes, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_linear_grad(const sllm_matrix* dy, const sllm_mx* w, const sllm_matrix* dx, void* workspace,
                                       uint64_t workspace_bytes, int32_t device, void* stream) try {
    clear_error();
    if (!dy) return fail(SLLM_E_INVAL, "dy: NULL");
    return linear(dy, nullptr, w, dx, true, workspace, workspace_bytes, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_linear_workspace(const sllm_matrix* x, const sllm_mx* w, uint64_t* bytes) try {
    clear_error();
    if (!x) return fail(SLLM_E_INVAL, "x: NULL");
    return linear_bytes(x, nullptr, w, false, bytes);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_linear_mx_workspace(const sllm_mx* x, const sllm_mx* w, uint64_t* bytes) try {
    clear_error();
    return linear_bytes(nullptr, x, w, false, bytes);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_linear_grad_workspace(const sllm_matrix* dy, const sllm_mx* w, uint64_t* bytes) try {
    clear_error();
    if (!dy) return fail(SLLM_E_INVAL, "dy: NULL");
    return linear_bytes(dy, nullptr, w, true, bytes);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_embedding(const sllm_matrix* table, const sllm_ids* ids, float scale, const sllm_matrix* out,
                                  int32_t device, void* stream) try {
    clear_error();
    if (!table) return fail(SLLM_E_INVAL, "table: NULL");
    return embedding(table, nullptr, ids, scale, out, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_embedding_mx(const sllm_mx* table, const sllm_ids* ids, float scale, const sllm_matrix* out,
                                     int32_t device, void* stream) try {
    clear_error();
    return embedding(nullptr, table, ids, scale, out, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_embedding_grad(const sllm_matrix* dy, const sllm_ids* ids, float scale, uint32_t flags,
                                       const sllm_matrix* grad, void* workspace, uint64_t workspace_bytes,
                                       int32_t device, void* stream) try {
    clear_error();
    Span s[4];
    SLLM_TRY(matrix_span("grad", grad, &s[0]));
    SLLM_TRY(matrix_span("dy", dy, &s[2]));
    SLLM_TRY(ids_span(ids, &s[3]));
    if (flags & ~SLLM_GRAD_ACCUMULATE) return fail(SLLM_E_INVAL, "unknown flags %#x", flags);
    if (dy->rows != ids->n || dy->cols != grad->cols)
        return fail(SLLM_E_INVAL, "dy is %llu x %llu, not %llu x %llu", (unsigned long long)dy->rows,
                    (unsigned long long)dy->cols, (unsigned long long)ids->n, (unsigned long long)grad->cols);
    if (ids->n > kMaxGradIds)
        return fail(SLLM_E_RANGE, "%llu ids, at most %llu", (unsigned long long)ids->n, (unsigned long long)kMaxGradIds);
    SLLM_TRY(workspace_span(workspace, workspace_bytes, embedding_grad_workspace(ids->n, grad->rows, grad->cols), &s[1]));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, 4, 2, device));
    EmbeddingGradLaunch a;
    a.dy = dy->data, a.dy_stride = dy->stride, a.dy_dtype = dy->dtype;
    a.ids = ids->data, a.ids64 = ids->bits == 64, a.n = ids->n;
    a.scale = scale;
    a.accumulate = flags & SLLM_GRAD_ACCUMULATE;
    a.grad = grad->data, a.grad_stride = grad->stride, a.grad_dtype = grad->dtype;
    a.vocab = grad->rows, a.dim = grad->cols;
    if (!a.vocab || !a.dim || (a.accumulate && !a.n)) return SLLM_OK;
    return launch_embedding_grad(a, workspace, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_embedding_grad_workspace(uint64_t n_ids, const sllm_matrix* grad, uint64_t* bytes) try {
    clear_error();
    Span s;
    SLLM_TRY(matrix_span("grad", grad, &s));
    if (!bytes) return fail(SLLM_E_INVAL, "bytes: NULL");
    if (n_ids > kMaxGradIds)
        return fail(SLLM_E_RANGE, "%llu ids, at most %llu", (unsigned long long)n_ids, (unsigned long long)kMaxGradIds);
    *bytes = embedding_grad_workspace(n_ids, grad->rows, grad->cols);
    return SLLM_OK;
}
SLLM_CATCH_ALL
