// gfx950 kernel of products with both sides in MX FP4.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStepBlocks = kNarrowStep / kMxBlock;

template <int BM, int BN, int WM, int WN, typename T>
__global__ __launch_bounds__(WM* WN * 64) void narrow_product(NarrowArgs a, T* out) {
    constexpr int kWaves = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kRowBytes = kNarrowStep / 2;
    // The two stages are variables of their own: the compiler then sees that
    // loads into one do not touch what is read from the other.
    __shared__ __align__(16) uint8_t lds_x0[BM * kRowBytes], lds_x1[BM * kRowBytes];
    __shared__ __align__(16) uint8_t lds_w0[BN * kRowBytes], lds_w1[BN * kRowBytes];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 15, g = lane >> 4;
    const void* const zeros = zero_vector();
    const uint64_t m0 = (uint64_t)blockIdx.x % a.tiles_m * BM, j0 = (uint64_t)blockIdx.x / a.tiles_m * BN;
    const uint32_t t0 = (uint64_t)a.steps * blockIdx.y / gridDim.y, t1 = (uint64_t)a.steps * (blockIdx.y + 1) / gridDim.y;
    const uint32_t wm = wave % WM, wn = wave / WM;

    f32x4 acc[FN][FM];
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[n][m] = f32x4{0, 0, 0, 0};

    // one load holds 16 rows x 4 blocks
    auto load = [&](uint32_t t, uint8_t* to_x, uint8_t* to_w) {
        const uint64_t b0 = (uint64_t)t * kStepBlocks;
#pragma unroll
        for (int q = 0; q < BM / 16 * 2 / kWaves; ++q) {
            const uint32_t at = q * kWaves + wave;
            const uint64_t row = min(m0 + at / 2 * 16 + r, a.m - 1), b = b0 + at % 2 * 4 + g;
            load_to_lds(b < a.blocks ? (const void*)(a.x_codes + row * a.blocks + b) : zeros, to_x + at * 1024);
        }
#pragma unroll
        for (int q = 0; q < BN / 16 * 2 / kWaves; ++q) {
            const uint32_t at = q * kWaves + wave;
            // past the end of the depth x is zero, so any finite values do
            const uint64_t row = min(j0 + at / 2 * 16 + r, a.n - 1), b = min(b0 + at % 2 * 4 + g, a.blocks - 1);
            load_to_lds(a.w_codes + row * a.blocks + b, to_w + at * 1024);
        }
    };
    // Lane (r, g) multiplies blocks 2 g and 2 g + 1 of its rows: two scale
    // bytes a row and stage.  Those past the row's end may hold anything.
    uint32_t xs[FM], ws[FN], mask = 0;
    auto load_scales = [&](uint32_t t) {
        const uint64_t b = (uint64_t)t * kStepBlocks + 2 * g;
        mask = b + 1 < a.blocks ? 0xffff : b < a.blocks ? 0xff : 0;
#pragma unroll
        for (int m = 0; m < FM; ++m) {
            const uint64_t row = min(m0 + (wm * FM + m) * 16 + r, a.m - 1);
            xs[m] = *reinterpret_cast<const uint16_t*>(a.x_scales + row * a.scale_pitch + b);
        }
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            const uint64_t row = min(j0 + (wn * FN + n) * 16 + r, a.n - 1);
            ws[n] = *reinterpret_cast<const uint16_t*>(a.w_scales + row * a.scale_pitch + b);
        }
    };
    const uint32_t x_at = wm * FM * 2048 + (g >> 1) * 1024 + (g & 1) * 512 + r * 16;
    const uint32_t w_at = wn * FN * 2048 + (g >> 1) * 1024 + (g & 1) * 512 + r * 16;
    auto stage = [&](uint32_t t, const uint8_t* x_now, uint8_t* x_next, const uint8_t* w_now, uint8_t* w_next) {
        wait_loads();
        __syncthreads();
        uint32_t x_scale[FM], w_scale[FN];
#pragma unroll
        for (int m = 0; m < FM; ++m) x_scale[m] = xs[m] & mask;
#pragma unroll
        for (int n = 0; n < FN; ++n) w_scale[n] = ws[n] & mask;
        if (t + 1 < t1) {
            load(t + 1, x_next, w_next);
            load_scales(t + 1);
        }
        auto half = [&](auto step) {
            constexpr int j = decltype(step)::value;
            u32x4 x[FM];
#pragma unroll
            for (int m = 0; m < FM; ++m) x[m] = *reinterpret_cast<const u32x4*>(x_now + (x_at + m * 2048 + j * 256));
#pragma unroll
            for (int n = 0; n < FN; ++n) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(w_now + (w_at + n * 2048 + j * 256));
#pragma unroll
                for (int m = 0; m < FM; ++m)
                    acc[n][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(w), fragment(x[m]), acc[n][m], 4, 4,
                                                                                 j, w_scale[n], j, x_scale[m]);
            }
        };
        half(std::integral_constant<int, 0>());
        half(std::integral_constant<int, 1>());
    };
    if (t0 < t1) {
        load(t0, lds_x0, lds_w0);
        load_scales(t0);
    }
    for (uint32_t t = t0; t < t1; t += 2) {
        stage(t, lds_x0, lds_x1, lds_w0, lds_w1);
        if (t + 1 < t1) stage(t + 1, lds_x1, lds_x0, lds_w1, lds_w0);
    }
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 16, j0 + wn * FN * 16, out);
}

}  // namespace

int32_t launch_narrow(const NarrowArgs& a, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, (narrow_product<256, 256, 2, 4, T><<<grid, 512, 0, stream>>>(a, static_cast<T*>(out))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
