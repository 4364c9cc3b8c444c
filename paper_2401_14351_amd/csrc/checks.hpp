// Checks of the operators' arguments that their entry points share.
#pragma once

#include "common.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

// A run of bytes an operator reads or writes.
struct Span {
    const char* name;
    const uint8_t* p;
    uint64_t bytes;
};

inline int32_t check_extent(const char* name, uint64_t rows, uint64_t cols) {
    if (rows > SLLM_MAX_EXTENT || cols > SLLM_MAX_EXTENT)
        return fail(SLLM_E_RANGE, "%s: %llu x %llu is larger than %llu rows or columns", name, (unsigned long long)rows,
                    (unsigned long long)cols, (unsigned long long)SLLM_MAX_EXTENT);
    return SLLM_OK;
}

inline int32_t check_pointer(const Span& s, uint64_t alignment) {
    if (!s.bytes) return SLLM_OK;
    if (!s.p) return fail(SLLM_E_INVAL, "%s: NULL pointer", s.name);
    if (reinterpret_cast<uintptr_t>(s.p) % alignment)
        return fail(SLLM_E_INVAL, "%s must be %llu-byte aligned", s.name, (unsigned long long)alignment);
    return SLLM_OK;
}

inline uint64_t itemsize(uint32_t dtype) { return dtype == SLLM_DTYPE_F32 ? 4 : 2; }

inline int32_t matrix_span(const char* name, const sllm_matrix* m, Span* out) {
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

inline int32_t mx_spans(const char* codes, const char* scales, const sllm_mx* m, Span* out, bool fp8 = false) {
    if (!m) return fail(SLLM_E_INVAL, "%s: NULL", codes);
    SLLM_TRY(check_extent(codes, m->rows, m->cols));
    out[0] = Span{codes, static_cast<const uint8_t*>(m->codes), m->rows * (fp8 ? mx8_code_pitch(m->cols) : mx_code_pitch(m->cols))};
    out[1] = Span{scales, static_cast<const uint8_t*>(m->scales), m->rows * mx_scale_pitch(m->cols)};
    SLLM_TRY(check_pointer(out[0], 16));
    return check_pointer(out[1], 16);
}

inline int32_t ids_span(const sllm_ids* ids, Span* out) {
    if (!ids) return fail(SLLM_E_INVAL, "ids: NULL");
    if (ids->bits != 32 && ids->bits != 64) return fail(SLLM_E_INVAL, "ids: %u bits, not 32 or 64", ids->bits);
    if (ids->reserved) return fail(SLLM_E_INVAL, "ids: reserved must be 0");
    SLLM_TRY(check_extent("ids", ids->n, 0));
    *out = Span{"ids", static_cast<const uint8_t*>(ids->data), ids->n * (ids->bits / 8)};
    return check_pointer(*out, ids->bits / 8);
}

// The first n_out spans, which are written, overlap no other.
inline int32_t check_overlaps(const Span* s, int n, int n_out) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n_out; ++j)
            if (i != j && s[i].bytes && s[j].bytes && s[i].p < s[j].p + s[j].bytes && s[j].p < s[i].p + s[i].bytes)
                return fail(SLLM_E_INVAL, "%s and %s overlap", s[i].name, s[j].name);
    return SLLM_OK;
}

// And all of them are device memory.
inline int32_t check_spans(const Span* s, int n, int n_out, int32_t device) {
    SLLM_TRY(check_overlaps(s, n, n_out));
    for (int i = 0; i < n; ++i) SLLM_TRY(check_device_range(s[i].p, s[i].bytes, device, s[i].name));
    return SLLM_OK;
}

inline int32_t workspace_span(void* workspace, uint64_t bytes, uint64_t need, Span* out) {
    if (bytes < need)
        return fail(SLLM_E_RANGE, "workspace of %llu bytes, %llu needed", (unsigned long long)bytes,
                    (unsigned long long)need);
    *out = Span{"workspace", static_cast<const uint8_t*>(workspace), need};
    return check_pointer(*out, 16);
}

}  // namespace sllm
