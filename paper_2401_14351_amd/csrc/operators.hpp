// Host-side launchers of the operators on loaded weights.  The entry points in
// operators.cpp have checked every argument: shapes agree, buffers are device
// memory and do not overlap, and no extent is past SLLM_MAX_EXTENT.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "sllm.h"

namespace sllm {

constexpr uint32_t kMxBlock = 32;       // columns that share a scale
constexpr uint32_t kMxBlockBytes = 16;  // their codes

inline uint64_t mx_blocks(uint64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }
inline uint64_t mx_code_pitch(uint64_t cols) { return mx_blocks(cols) * kMxBlockBytes; }
inline uint64_t mx_scale_pitch(uint64_t cols) { return (mx_blocks(cols) + 15) / 16 * 16; }

// One operand of a product: a matrix, or one in MX FP4 (codes set).
struct Operand {
    const void* data = nullptr;
    uint64_t stride = 0;
    uint32_t dtype = 0;
    const uint8_t* codes = nullptr;
    const uint8_t* scales = nullptr;
};

// out (m x n) = x (m x k) * transpose(w), w in MX FP4 n x k; or, with `grad`,
// out (m x k) = x (m x n) * w.
struct LinearLaunch {
    uint64_t m = 0, n = 0, k = 0;
    Operand x;
    const uint8_t* w_codes = nullptr;
    const uint8_t* w_scales = nullptr;
    void* out = nullptr;
    uint64_t out_stride = 0;
    uint32_t out_dtype = 0;
    bool grad = false;
};
uint64_t linear_workspace(const LinearLaunch& a);
int32_t launch_linear(const LinearLaunch& a, void* workspace, hipStream_t stream);

int32_t launch_quantize(const sllm_matrix& src, const sllm_mx& dst, hipStream_t stream);

// out's row i = scale * table row ids[i], zeros where there is none; ids null:
// row i itself, not scaled.
struct EmbeddingLaunch {
    Operand table;
    uint64_t vocab = 0, dim = 0;
    const void* ids = nullptr;
    bool ids64 = false;
    uint64_t n = 0;
    float scale = 1.0f;
    void* out = nullptr;
    uint64_t out_stride = 0;
    uint32_t out_dtype = 0;
};
int32_t launch_embedding(const EmbeddingLaunch& a, hipStream_t stream);

struct EmbeddingGradLaunch {
    const void* dy = nullptr;
    uint64_t dy_stride = 0;
    uint32_t dy_dtype = 0;
    const void* ids = nullptr;
    bool ids64 = false;
    uint64_t n = 0;
    float scale = 1.0f;
    bool accumulate = false;
    void* grad = nullptr;
    uint64_t vocab = 0, dim = 0, grad_stride = 0;
    uint32_t grad_dtype = 0;
};
constexpr uint64_t kMaxGradIds = 1ull << 24;
uint64_t embedding_grad_workspace(uint64_t n_ids, uint64_t vocab, uint64_t dim);
int32_t launch_embedding_grad(const EmbeddingGradLaunch& a, void* workspace, hipStream_t stream);

}  // namespace sllm
