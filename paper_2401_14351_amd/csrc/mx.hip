// gfx950 kernels of MX FP4 matrices: quantisation and products.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

namespace {

// ---------------------------------------------------------------------------
// Quantisation
// ---------------------------------------------------------------------------

// The scale byte of a block whose largest magnitude is `top` (0 to 254, or 255
// where it is no finite number): floor(log2 top) is the float's exponent
// field less 127, two less make 4 .. 8 of the largest element, and magnitudes
// below 2^-125 share the smallest scale.
__device__ __forceinline__ uint32_t block_scale(float top) {
    const uint32_t e = __float_as_uint(top) >> 23;
    return e == 255 ? 255 : e < 2 ? 0 : e - 2;
}

// One lane per block.
template <typename T>
__global__ __launch_bounds__(256) void mx_quantize(const T* src, uint64_t stride, uint64_t rows, uint32_t cols,
                                                   uint32_t scale_pitch, uint8_t* codes, uint8_t* scales) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint64_t row = i / scale_pitch;
    const uint32_t b = i % scale_pitch, blocks = (cols + 31) / 32;
    if (row >= rows) return;
    if (b >= blocks) {
        scales[row * scale_pitch + b] = 0;
        return;
    }
    float v[32], top = 0;
    bool finite = true;
    for (uint32_t c = 0; c < 32; ++c) {
        v[c] = b * 32 + c < cols ? to_f32(src[row * stride + b * 32 + c]) : 0.0f;
        finite &= (__float_as_uint(v[c]) & 0x7f800000) != 0x7f800000;
        top = fmaxf(top, fabsf(v[c]));
    }
    const uint32_t s = finite ? block_scale(top) : 255;
    u32x4 out = {0, 0, 0, 0};
    if (finite)
        for (uint32_t c = 0; c < 32; c += 2) {
            const uint32_t two = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[c], v[c + 1], mx_scale(s), 0) & 0xff;
            out[c / 8] |= two << (c % 8 * 4);
        }
    reinterpret_cast<u32x4*>(codes)[row * blocks + b] = out;
    scales[row * scale_pitch + b] = s;
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

struct Product {
    Operand x;
    const uint8_t* w_codes;
    const uint8_t* w_scales;
    uint64_t m, n, k;
    uint64_t x_cols;
    void* out;
    uint64_t out_stride;
    uint32_t out_dtype;
};

__device__ float mx_at(const uint8_t* codes, const uint8_t* scales, uint64_t cols, uint64_t r, uint64_t c) {
    const uint64_t blocks = (cols + 31) / 32, pitch = (blocks + 15) / 16 * 16;
    return mx_value(codes[r * blocks * 16 + c / 2], c & 1, scales[r * pitch + c / 32]);
}

// A tile of 32 x 32 outputs a workgroup, 32 steps of the sum at a time through LDS.
template <bool Grad>
__global__ __launch_bounds__(256) void mx_product(Product p) {
    __shared__ float xs[32][33], ws[32][33];
    const uint64_t cols = Grad ? p.k : p.n, depth = Grad ? p.n : p.k;
    const uint64_t m0 = (uint64_t)blockIdx.y * 32, j0 = (uint64_t)blockIdx.x * 32;
    const uint32_t tx = threadIdx.x % 32, ty = threadIdx.x / 32;
    float acc[4] = {0, 0, 0, 0};
    for (uint64_t d0 = 0; d0 < depth; d0 += 32) {
        for (uint32_t r = ty; r < 32; r += 8) {
            const uint64_t m = m0 + r, d = d0 + tx;
            float v = 0;
            if (m < p.m && d < depth) {
                if (p.x.codes)
                    v = mx_at(p.x.codes, p.x.scales, p.x_cols, m, d);
                else if (p.x.dtype == SLLM_DTYPE_F32)
                    v = static_cast<const float*>(p.x.data)[m * p.x.stride + d];
                else if (p.x.dtype == SLLM_DTYPE_F16)
                    v = to_f32(static_cast<const _Float16*>(p.x.data)[m * p.x.stride + d]);
                else
                    v = to_f32(static_cast<const __bf16*>(p.x.data)[m * p.x.stride + d]);
            }
            xs[r][tx] = v;
            // ws[d][j]
            const uint64_t n = Grad ? d0 + r : j0 + r, k = Grad ? j0 + tx : d0 + tx;
            const float w = n < p.n && k < p.k ? mx_at(p.w_codes, p.w_scales, p.k, n, k) : 0.0f;
            if (Grad)
                ws[r][tx] = w;
            else
                ws[tx][r] = w;
        }
        __syncthreads();
        for (uint32_t d = 0; d < 32; ++d)
            for (uint32_t i = 0; i < 4; ++i) acc[i] += xs[ty + 8 * i][d] * ws[d][tx];
        __syncthreads();
    }
    for (uint32_t i = 0; i < 4; ++i) {
        const uint64_t m = m0 + ty + 8 * i, j = j0 + tx;
        if (m >= p.m || j >= cols) continue;
        const uint64_t at = m * p.out_stride + j;
        if (p.out_dtype == SLLM_DTYPE_F32)
            static_cast<float*>(p.out)[at] = acc[i];
        else if (p.out_dtype == SLLM_DTYPE_F16)
            static_cast<_Float16*>(p.out)[at] = from_f32<_Float16>(acc[i]);
        else
            static_cast<__bf16*>(p.out)[at] = from_f32<__bf16>(acc[i]);
    }
}

}  // namespace

int32_t launch_quantize(const sllm_matrix& src, const sllm_mx& dst, hipStream_t stream) {
    const uint32_t pitch = (uint32_t)mx_scale_pitch(src.cols);
    const uint64_t grid = ceil_div(src.rows * pitch, 256);
    if (grid > UINT32_MAX / 256) return fail(SLLM_E_RANGE, "matrix too large");
    SLLM_BY_DTYPE(src.dtype, T,
                  mx_quantize<T><<<(uint32_t)grid, 256, 0, stream>>>(
                      static_cast<const T*>(src.data), src.stride, src.rows, (uint32_t)src.cols, pitch,
                      static_cast<uint8_t*>(dst.codes), static_cast<uint8_t*>(dst.scales)));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

uint64_t linear_workspace(const LinearLaunch& a) { return 0; }

int32_t launch_linear(const LinearLaunch& a, void* workspace, hipStream_t stream) {
    const Product p{a.x, a.w_codes, a.w_scales, a.m, a.n, a.k, a.grad ? a.n : a.k, a.out, a.out_stride, a.out_dtype};
    const uint64_t gx = ceil_div(a.grad ? a.k : a.n, 32), gy = ceil_div(a.m, 32);
    if (gx > UINT32_MAX / 256 || gy > 65535) return fail(SLLM_E_RANGE, "product too large");
    const dim3 grid((uint32_t)gx, (uint32_t)gy);
    if (a.grad)
        mx_product<true><<<grid, 256, 0, stream>>>(p);
    else
        mx_product<false><<<grid, 256, 0, stream>>>(p);
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
