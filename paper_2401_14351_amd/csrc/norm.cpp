// Entry points of norms and of matrices in MX FP8: argument checks, then the launchers of
// norm.hip.
#include <cmath>

#include "checks.hpp"
#include "common.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

namespace {

int32_t same_matrix(const char* name, const sllm_matrix& m, const sllm_matrix& like) {
    if (m.rows != like.rows || m.cols != like.cols || m.dtype != like.dtype)
        return fail(SLLM_E_INVAL, "%s is %llu x %llu of dtype %u, not %llu x %llu of dtype %u", name, (unsigned long long)m.rows,
                    (unsigned long long)m.cols, m.dtype, (unsigned long long)like.rows, (unsigned long long)like.cols, like.dtype);
    return SLLM_OK;
}

int32_t gain_span(const char* name, const sllm_matrix* gain, uint64_t cols, Span* out) {
    SLLM_TRY(matrix_span(name, gain, out));
    if (gain->rows != 1 || gain->cols != cols)
        return fail(SLLM_E_INVAL, "%s is %llu x %llu, not 1 x %llu", name, (unsigned long long)gain->rows, (unsigned long long)gain->cols,
                    (unsigned long long)cols);
    return SLLM_OK;
}

int32_t floats_span(const char* name, const float* p, uint64_t n, Span* out) {
    *out = Span{name, reinterpret_cast<const uint8_t*>(p), p ? n * 4 : 0};
    return check_pointer(*out, 4);
}

int32_t norm(const sllm_matrix* x, const sllm_matrix* residual, const sllm_matrix* gain, float eps, const sllm_matrix* h, const sllm_matrix* y,
             const sllm_mx* y8, float* inverse, int32_t device, void* stream) {
    NormLaunch a;
    Span s[7];
    int n = 0;
    if (y8) {
        SLLM_TRY(mx_spans("y codes", "y scales", y8, s, true));
        n = 2;
    } else {
        SLLM_TRY(matrix_span("y", y, &s[n++]));
    }
    SLLM_TRY(matrix_span("x", x, &s[n]));
    const Span x_span = s[n];
    SLLM_TRY(floats_span("inverse", inverse, x->rows, &s[n++]));
    if (!h != !residual) return fail(SLLM_E_INVAL, "h goes with a residual");
    if (h) {
        SLLM_TRY(matrix_span("h", h, &s[n++]));
        SLLM_TRY(same_matrix("h", *h, *x));
    }
    const int n_out = n;
    s[n++] = x_span;
    if (residual) {
        SLLM_TRY(matrix_span("residual", residual, &s[n++]));
        SLLM_TRY(same_matrix("residual", *residual, *x));
        a.residual = residual->data, a.residual_stride = residual->stride;
        a.h = h->data, a.h_stride = h->stride;
    }
    SLLM_TRY(gain_span("gain", gain, x->cols, &s[n++]));
    if (y8) {
        if (y8->rows != x->rows || y8->cols != x->cols) return fail(SLLM_E_INVAL, "x and y differ in shape");
        a.codes = static_cast<uint8_t*>(y8->codes), a.scales = static_cast<uint8_t*>(y8->scales);
    } else {
        SLLM_TRY(same_matrix("y", *y, *x));
        a.y = y->data, a.y_stride = y->stride;
    }
    if (!(eps >= 0) || !std::isfinite(eps)) return fail(SLLM_E_INVAL, "eps %g is negative or no number", eps);
    a.x = x->data, a.x_stride = x->stride;
    a.gain = gain->data, a.gain_dtype = gain->dtype;
    a.rows = x->rows, a.cols = x->cols, a.dtype = x->dtype;
    a.eps = eps;
    a.inverse = inverse;
    SLLM_TRY(check_overlaps(s, n, n_out));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, n, n_out, device));
    if (!a.rows || !a.cols) return SLLM_OK;
    return launch_rms_norm(a, static_cast<hipStream_t>(stream));
}

}  // namespace

}  // namespace sllm

using namespace sllm;

extern "C" int32_t sllm_rms_norm(const sllm_matrix* x, const sllm_matrix* residual, const sllm_matrix* gain, float eps, const sllm_matrix* h,
                                 const sllm_matrix* y, float* inverse, int32_t device, void* stream) try {
    clear_error();
    return norm(x, residual, gain, eps, h, y, nullptr, inverse, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_rms_norm_octet(const sllm_matrix* x, const sllm_matrix* residual, const sllm_matrix* gain, float eps, const sllm_matrix* h,
                                     const sllm_mx* y, int32_t device, void* stream) try {
    clear_error();
    if (!y) return fail(SLLM_E_INVAL, "y: NULL");
    return norm(x, residual, gain, eps, h, nullptr, y, nullptr, device, stream);
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_rms_norm_grad(const sllm_matrix* dy, const sllm_matrix* dh, const sllm_matrix* h, const sllm_matrix* gain,
                                      const float* inverse, const sllm_matrix* dx, const sllm_matrix* dgain, void* workspace,
                                      uint64_t workspace_bytes, int32_t device, void* stream) try {
    clear_error();
    Span s[8];
    int n = 0;
    SLLM_TRY(matrix_span("dx", dx, &s[n++]));
    SLLM_TRY(gain_span("dgain", dgain, dx->cols, &s[n++]));
    SLLM_TRY(workspace_span(workspace, workspace_bytes, rms_norm_grad_workspace(dx->rows, dx->cols), &s[n++]));
    SLLM_TRY(matrix_span("dy", dy, &s[n++]));
    SLLM_TRY(matrix_span("h", h, &s[n++]));
    SLLM_TRY(gain_span("gain", gain, dx->cols, &s[n++]));
    if (!inverse && dx->rows) return fail(SLLM_E_INVAL, "inverse: NULL");
    SLLM_TRY(floats_span("inverse", inverse, dx->rows, &s[n++]));
    SLLM_TRY(same_matrix("dy", *dy, *dx));
    SLLM_TRY(same_matrix("h", *h, *dx));
    if (dgain->dtype != gain->dtype) return fail(SLLM_E_INVAL, "gain and its gradient differ in dtype");
    NormGradLaunch a;
    if (dh) {
        SLLM_TRY(matrix_span("dh", dh, &s[n++]));
        SLLM_TRY(same_matrix("dh", *dh, *dx));
        a.dh = dh->data, a.dh_stride = dh->stride;
    }
    a.dy = dy->data, a.dy_stride = dy->stride;
    a.h = h->data, a.h_stride = h->stride;
    a.gain = gain->data, a.gain_dtype = gain->dtype;
    a.rows = dx->rows, a.cols = dx->cols, a.dtype = dx->dtype;
    a.inverse = inverse;
    a.dx = dx->data, a.dx_stride = dx->stride;
    a.dgain = dgain->data;
    SLLM_TRY(check_overlaps(s, n, 3));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, n, 3, device));
    if (!a.cols) return SLLM_OK;
    return launch_rms_norm_grad(a, workspace, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_rms_norm_grad_workspace(uint64_t rows, uint64_t cols, uint64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(SLLM_E_INVAL, "bytes: NULL");
    SLLM_TRY(check_extent("rows", rows, cols));
    *bytes = rms_norm_grad_workspace(rows, cols);
    return SLLM_OK;
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_octet_sizes(uint64_t rows, uint64_t cols, uint64_t* codes_bytes, uint64_t* scales_bytes) try {
    clear_error();
    if (!codes_bytes || !scales_bytes) return fail(SLLM_E_INVAL, "codes_bytes and scales_bytes must be non-NULL");
    SLLM_TRY(check_extent("matrix", rows, cols));
    *codes_bytes = rows * mx8_code_pitch(cols);
    *scales_bytes = rows * mx_scale_pitch(cols);
    return SLLM_OK;
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_octet_quantize(const sllm_matrix* src, const sllm_mx* dst, int32_t device, void* stream) try {
    clear_error();
    Span s[3];
    SLLM_TRY(mx_spans("codes", "scales", dst, s, true));
    SLLM_TRY(matrix_span("source", src, &s[2]));
    if (src->rows != dst->rows || src->cols != dst->cols) return fail(SLLM_E_INVAL, "source and destination differ in shape");
    SLLM_TRY(check_overlaps(s, 3, 2));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, 3, 2, device));
    if (!src->rows || !src->cols) return SLLM_OK;
    return launch_mx8_quantize(*src, *dst, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_mx_octet_dequantize(const sllm_mx* src, const sllm_matrix* dst, int32_t device, void* stream) try {
    clear_error();
    Span s[3];
    SLLM_TRY(matrix_span("destination", dst, &s[0]));
    SLLM_TRY(mx_spans("codes", "scales", src, &s[1], true));
    if (src->rows != dst->rows || src->cols != dst->cols) return fail(SLLM_E_INVAL, "source and destination differ in shape");
    SLLM_TRY(check_overlaps(s, 3, 1));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, 3, 1, device));
    if (!src->rows || !src->cols) return SLLM_OK;
    return launch_mx8_dequantize(*src, *dst, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL
