// gfx950 kernels of products with few rows of x and an MX FP4 weight: decoding.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

// Eight elements of x as the bfloat16 vectors whose sum they are.
template <typename X>
struct Parts {
    static constexpr int n = sizeof(X) == 4 ? 3 : 2;
    bf16x8 v[n];

    __device__ __forceinline__ static Parts of(const X (&x)[8]) {
        Parts p;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = to_f32(x[e]);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t h = leading_bf16(f[e]);
                o[e / 2] = e % 2 ? o[e / 2] | h << 16 : h;
            }
            p.v[i] = __builtin_bit_cast(bf16x8, o);
        }
        return p;
    }
};

template <>
struct Parts<__bf16> {
    static constexpr int n = 1;
    bf16x8 v[1];

    __device__ __forceinline__ static Parts of(const __bf16 (&x)[8]) {
        Parts p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p.v[0][e] = x[e];
        return p;
    }
};

// Eight elements of a row from column c; those past the end are zero.
template <typename X>
__device__ __forceinline__ Parts<X> load_x(const X* row, uint64_t c, uint64_t cols) {
    X x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = c + e < cols ? row[c + e] : (X)0.0f;
    return Parts<X>::of(x);
}

template <typename X>
__device__ __forceinline__ Parts<X> load_x_vector(const X* p) {
    X x[8];
    constexpr int kVectors = sizeof(X) / 2;
    u32x4 v[kVectors];
#pragma unroll
    for (int i = 0; i < kVectors; ++i) v[i] = reinterpret_cast<const u32x4*>(p)[i];
    __builtin_memcpy(x, v, sizeof x);
    return Parts<X>::of(x);
}

// A workgroup makes 16 NT columns of the output, its waves each a run of the
// depth; their sums are joined in LDS, first to last.  Of a step of 128 of the
// depth, lane (r, g) holds block g of row r: the order in which the matrix
// instructions take a block's columns does not matter as long as both sides
// have the same.
template <typename X, int MT, int NT>
__global__ __launch_bounds__(1024) void skinny_product(SkinnyArgs a) {
    extern __shared__ float sums[];
    constexpr bool kMx = __is_same(X, void);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t waves = blockDim.x >> 6, r = lane & 15, g = lane >> 4;
    const uint64_t j0 = (uint64_t)blockIdx.x * 16 * NT;
    const uint32_t s0 = (uint64_t)a.steps * wave / waves, s1 = (uint64_t)a.steps * (wave + 1) / waves;

    f32x4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0, 0, 0, 0};

    const u32x4* w_codes[NT];
    const uint8_t* w_scales[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint64_t row = min(j0 + n * 16 + r, a.n - 1);
        w_codes[n] = a.w_codes + row * a.blocks;
        w_scales[n] = a.w_scales + row * a.scale_pitch;
    }
    uint64_t x_row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) x_row[m] = min((uint64_t)m * 16 + r, a.m - 1);

    // Kept steps of the weight are loaded ahead of the ones at work.
    constexpr uint32_t kAhead = 4;
    struct Weight {
        u32x4 codes[kAhead][NT];
        uint32_t scale[kAhead][NT];
    };
    // Blocks past the row's or the run's end: x is zero there, the scale must be a number.
    const uint64_t end = min(a.blocks, 4 * (uint64_t)s1);
    auto load_w = [&](uint32_t s) {
        Weight w;
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
            const uint64_t b = 4 * ((uint64_t)s + u) + g, at = min(b, a.blocks - 1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                w.codes[u][n] = w_codes[n][at];
                w.scale[u][n] = w_scales[n][at];
            }
        }
        return w;
    };
    Weight ahead = load_w(s0);
    if constexpr (kMx) {
        for (uint32_t s = s0; s < s1; s += kAhead) {
            const Weight w = ahead;
            u32x4 x[kAhead][MT];
            uint32_t xs[kAhead][MT];
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint64_t b = 4 * ((uint64_t)s + u) + g, at = min(b, a.blocks - 1);
                    x[u][m] = static_cast<const u32x4*>(a.x)[x_row[m] * a.blocks + at];
                    xs[u][m] = a.x_scales[x_row[m] * a.scale_pitch + at];
                }
            if (s + kAhead < s1) ahead = load_w(s + kAhead);
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                const uint32_t mask = 4 * ((uint64_t)s + u) + g < end ? ~0u : 0;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                            fragment(w.codes[u][n]), fragment(x[u][m] & mask), acc[m][n], 4, 4, 0, w.scale[u][n] & mask, 0,
                            xs[u][m] & mask);
            }
        }
    } else {
        const X* x[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) x[m] = static_cast<const X*>(a.x) + x_row[m] * a.x_stride;
        auto step = [&](const u32x4 (&codes)[NT], const uint32_t (&scale)[NT], uint64_t b, auto load) {
            u32x4 w[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) expand(codes[n], b < a.blocks ? scale[n] : 0, w[n]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const Parts<X> p = load(x[m], b * 32 + j * 8);
#pragma unroll
                    for (int i = 0; i < Parts<X>::n; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[n][j]), p.v[i],
                                                                                acc[m][n], 0, 0, 0);
                }
        };
        for (uint32_t s = s0; s < s1; s += kAhead) {
            const Weight w = ahead;
            if (s + kAhead < s1) ahead = load_w(s + kAhead);
            if (a.vector && (uint64_t)(s + kAhead) * 128 <= a.depth) {
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u)
                    if (s + u < s1)
                        step(w.codes[u], w.scale[u], 4 * ((uint64_t)s + u) + g, [](const X* row, uint64_t c) { return load_x_vector(row + c); });
            } else {
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u)
                    if (s + u < s1)
                        step(w.codes[u], w.scale[u], 4 * ((uint64_t)s + u) + g, [&](const X* row, uint64_t c) {
                            return a.vector && c + 8 <= a.depth ? load_x_vector(row + c) : load_x(row, c, a.depth);
                        });
            }
        }
    }

    // lane (r, g) has columns 4 g .. + 3 of the tile for row r of x
    constexpr uint32_t kCols = 16 * NT, kSums = 16 * MT * kCols;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
            *reinterpret_cast<f32x4*>(sums + wave * kSums + (m * 16 + r) * kCols + n * 16 + g * 4) = acc[m][n];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kSums; i += blockDim.x) {
        const uint64_t m = i / kCols, j = j0 + i % kCols;
        if (m >= a.m || j >= a.n) continue;
        float sum = 0;
        for (uint32_t w = 0; w < waves; ++w) sum += sums[w * kSums + i];
        const uint64_t at = m * a.out_stride + j;
        if (a.out_dtype == SLLM_DTYPE_F32)
            static_cast<float*>(a.out)[at] = sum;
        else if (a.out_dtype == SLLM_DTYPE_F16)
            static_cast<_Float16*>(a.out)[at] = from_f32<_Float16>(sum);
        else
            static_cast<__bf16*>(a.out)[at] = from_f32<__bf16>(sum);
    }
}

template <typename X, int MT, int NT>
void launch(const SkinnyArgs& a, hipStream_t stream) {
    const uint32_t grid = (uint32_t)((a.n + 16 * NT - 1) / (16 * NT));
    // enough waves to fill the GPU, but two steps of the depth for each
    uint32_t waves = 4;
    while (waves < 16 && grid * waves < 2048 && a.steps >= waves * 4) waves *= 2;
    while (waves > 1 && a.steps < waves) waves /= 2;
    skinny_product<X, MT, NT><<<grid, waves * 64, waves * 16 * MT * 16 * NT * 4, stream>>>(a);
}

template <typename X>
void launch_rows(const SkinnyArgs& a, hipStream_t stream) {
    if (a.m <= 16)
        launch<X, 1, 1>(a, stream);
    else
        launch<X, 2, 1>(a, stream);
}

}  // namespace

int32_t launch_skinny(const SkinnyArgs& a, hipStream_t stream) {
    if (a.x_scales)
        launch_rows<void>(a, stream);
    else
        SLLM_BY_DTYPE(a.x_dtype, X, launch_rows<X>(a, stream));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
