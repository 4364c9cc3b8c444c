// gfx950 kernels of token embeddings: the lookup of table rows (and the
// dequantisation of a whole matrix, a lookup of every row in turn) and its
// gradient.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

namespace {

struct Ids {
    const void* p;
    bool wide;
};

// Id i, or -1 where it names none of `vocab` rows.
__device__ __forceinline__ int32_t id_at(const Ids& ids, uint64_t i, uint32_t vocab) {
    const int64_t v = ids.wide ? static_cast<const int64_t*>(ids.p)[i] : static_cast<const int32_t*>(ids.p)[i];
    return v < 0 || v >= (int64_t)vocab ? -1 : (int32_t)v;
}

struct Lookup {
    Operand table;
    uint32_t vocab, dim;
    Ids ids;
    uint64_t n;
    float scale;
    uint64_t out_stride;
};

// A workgroup per row.  S: the table's elements, void for MX FP4.
template <typename S, typename T>
__global__ __launch_bounds__(256) void lookup(Lookup a, T* out) {
    for (uint64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
        const int64_t row = a.ids.p ? id_at(a.ids, i, a.vocab) : (int64_t)i;
        for (uint32_t c = threadIdx.x; c < a.dim; c += 256) {
            float v = 0;
            if (row >= 0) {
                if constexpr (__is_same(S, void)) {
                    const uint32_t blocks = (a.dim + 31) / 32, pitch = (blocks + 15) / 16 * 16;
                    v = mx_value(a.table.codes[(uint64_t)row * blocks * 16 + c / 2], c & 1,
                                 a.table.scales[(uint64_t)row * pitch + c / 32]);
                } else {
                    v = to_f32(static_cast<const S*>(a.table.data)[row * a.table.stride + c]);
                }
            }
            out[i * a.out_stride + c] = from_f32<T>(v * a.scale);
        }
    }
}

struct GradArgs {
    uint64_t dy_stride;
    Ids ids;
    uint64_t n;
    float scale;
    uint32_t vocab, dim;
    uint64_t grad_stride;
    bool accumulate;
};

// A workgroup per table row goes through all ids.
template <typename S, typename T>
__global__ __launch_bounds__(256) void gather_grad(GradArgs a, const S* dy, T* grad) {
    for (uint32_t row = blockIdx.x; row < a.vocab; row += gridDim.x)
        for (uint32_t c = threadIdx.x; c < a.dim; c += 256) {
            float sum = 0;
            bool any = false;
            for (uint64_t i = 0; i < a.n; ++i)
                if (id_at(a.ids, i, a.vocab) == (int32_t)row) {
                    sum += to_f32(dy[i * a.dy_stride + c]);
                    any = true;
                }
            const uint64_t at = (uint64_t)row * a.grad_stride + c;
            sum *= a.scale;
            if (a.accumulate && any) grad[at] = from_f32<T>(to_f32(grad[at]) + sum);
            if (!a.accumulate) grad[at] = from_f32<T>(sum);
        }
}

}  // namespace

int32_t launch_embedding(const EmbeddingLaunch& a, hipStream_t stream) {
    const Lookup l{a.table, (uint32_t)a.vocab, (uint32_t)a.dim, {a.ids, a.ids64}, a.n, a.scale, a.out_stride};
    const uint32_t grid = (uint32_t)std::min<uint64_t>(a.n, 1u << 20);
    SLLM_BY_DTYPE(a.out_dtype, T, {
        T* out = static_cast<T*>(a.out);
        if (a.table.codes)
            lookup<void, T><<<grid, 256, 0, stream>>>(l, out);
        else
            SLLM_BY_DTYPE(a.table.dtype, S, (lookup<S, T><<<grid, 256, 0, stream>>>(l, out)));
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

uint64_t embedding_grad_workspace(uint64_t n_ids, uint64_t vocab, uint64_t dim) { return 0; }

int32_t launch_embedding_grad(const EmbeddingGradLaunch& a, void* workspace, hipStream_t stream) {
    const GradArgs g{a.dy_stride, {a.ids, a.ids64}, a.n, a.scale, (uint32_t)a.vocab, (uint32_t)a.dim, a.grad_stride,
                     a.accumulate};
    const uint32_t grid = (uint32_t)std::min<uint64_t>(a.vocab, 1u << 20);
    SLLM_BY_DTYPE(a.dy_dtype, S, SLLM_BY_DTYPE(a.grad_dtype, T, (gather_grad<S, T><<<grid, 256, 0, stream>>>(
                                                                    g, static_cast<const S*>(a.dy),
                                                                    static_cast<T*>(a.grad)))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
