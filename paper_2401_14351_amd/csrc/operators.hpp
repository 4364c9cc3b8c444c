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
inline uint64_t mx8_code_pitch(uint64_t cols) { return mx_blocks(cols) * kMxBlock; }
inline uint64_t mx_scale_pitch(uint64_t cols) { return (mx_blocks(cols) + 15) / 16 * 16; }

// One operand of a product: a matrix, or one in MX FP4 or FP8 (codes set).
struct Operand {
    const void* data = nullptr;
    uint64_t stride = 0;
    uint32_t dtype = 0;
    const uint8_t* codes = nullptr;
    const uint8_t* scales = nullptr;
    bool fp8 = false;
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

// h = x + residual (h = x where there is none); y = h / sqrt(mean h^2 + eps) * gain, as a
// matrix or in MX FP8 (codes set).
struct NormLaunch {
    const void *x = nullptr, *residual = nullptr, *gain = nullptr;
    uint64_t x_stride = 0, residual_stride = 0, rows = 0, cols = 0;
    uint32_t dtype = 0, gain_dtype = 0;
    float eps = 0;
    void *h = nullptr, *y = nullptr;
    uint64_t h_stride = 0, y_stride = 0;
    float* inverse = nullptr;  // of each row's root mean square, if not null
    uint8_t *codes = nullptr, *scales = nullptr;
};
int32_t launch_rms_norm(const NormLaunch& a, hipStream_t stream);

struct NormGradLaunch {
    const void *dy = nullptr, *dh = nullptr, *h = nullptr, *gain = nullptr;
    uint64_t dy_stride = 0, dh_stride = 0, h_stride = 0, rows = 0, cols = 0;
    uint32_t dtype = 0, gain_dtype = 0;
    const float* inverse = nullptr;
    void *dx = nullptr, *dgain = nullptr;
    uint64_t dx_stride = 0;
};
uint64_t rms_norm_grad_workspace(uint64_t rows, uint64_t cols);
int32_t launch_rms_norm_grad(const NormGradLaunch& a, void* workspace, hipStream_t stream);

int32_t launch_mx8_quantize(const sllm_matrix& src, const sllm_mx& dst, hipStream_t stream);
int32_t launch_mx8_dequantize(const sllm_mx& src, const sllm_matrix& dst, hipStream_t stream);

// Causal attention of packed sequences, or behind what a cache holds of them (cache_k set).
// Strides are in elements; window, sinks and tokens are below 2^30.
struct AttentionArgs {
    const void *q = nullptr, *k = nullptr, *v = nullptr;
    uint64_t q_token = 0, q_head = 0, k_token = 0, k_head = 0, v_token = 0, v_head = 0;
    void* out = nullptr;
    uint64_t out_token = 0, out_head = 0;
    float* lse = nullptr;  // tokens x heads
    uint32_t tokens = 0, heads = 0, kv_heads = 0, group = 0, dim = 0, dtype = 0;
    int32_t window = 0, sinks = 0;
    float scale = 0;
    const void* offsets = nullptr;  // sequences + 1, or null for one sequence
    uint32_t sequences = 0;
    bool wide_offsets = false, wide_lengths = false;
    bool vec = false;  // rows start on 16 bytes and are whole multiples of them
    const void* lengths = nullptr;
    void *cache_k = nullptr, *cache_v = nullptr;  // (sequences, kv_heads, slots, dim)
    uint64_t slots = 0;
    uint32_t pieces = 0;   // of each key/value head
    uint32_t element = 0;  // bytes
};
int32_t launch_attention(AttentionArgs a, hipStream_t stream);

struct AttentionGradArgs : AttentionArgs {  // out is read
    const void* dout = nullptr;
    uint64_t dout_token = 0, dout_head = 0;
    void *dq = nullptr, *dk = nullptr, *dv = nullptr;
    uint64_t dq_token = 0, dq_head = 0, dk_token = 0, dk_head = 0, dv_token = 0, dv_head = 0;
    float* rows = nullptr;  // tokens x heads, three times
    uint32_t splits = 1;    // of the rows that see a key
    float* parts = nullptr;
    // what rows behind the window give to sinks: in so many parts, rows of sinks in each, by
    // their place among the tokens or by sequence, and tiles of sinks of a sequence (0: of any)
    uint32_t far = 0;
    uint64_t far_rows = 0;
    bool far_packed = false;
    uint32_t sink_tiles = 0;
    float* far_parts = nullptr;
};
uint64_t attention_grad_workspace(AttentionGradArgs a);
int32_t launch_attention_grad(AttentionGradArgs a, void* workspace, hipStream_t stream);

// One new token a sequence, tokens and sequences being the same.
uint64_t attention_step_workspace(const AttentionArgs& a);
int32_t launch_attention_step(const AttentionArgs& a, void* workspace, hipStream_t stream);

}  // namespace sllm
