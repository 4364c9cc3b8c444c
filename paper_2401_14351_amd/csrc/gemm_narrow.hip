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
    // scales of two stages: 16 bytes a row, x's rows then w's
    __shared__ __align__(16) uint8_t lds_s0[(BM + BN) * 16], lds_s1[(BM + BN) * 16];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 15, g = lane >> 4;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    const uint32_t wm = wave % WM, wn = wave / WM;
    // splits begin at pairs of stages, which share their scales
    const uint32_t pairs = (a.steps + 1) / 2;
    const uint32_t t0 = (uint64_t)pairs * blockIdx.y / gridDim.y * 2;
    const uint32_t t1 = min((uint32_t)((uint64_t)pairs * (blockIdx.y + 1) / gridDim.y * 2), a.steps);

    f32x4 acc[FN][FM];
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[n][m] = f32x4{0, 0, 0, 0};

    // one load holds 8 rows x 8 blocks
    auto load = [&](uint32_t t, uint8_t* to_x, uint8_t* to_w) {
        const uint64_t b0 = (uint64_t)t * kStepBlocks;
#pragma unroll
        for (int q = 0; q < BM / 8 / kWaves; ++q) {
            const uint32_t at = q * kWaves + wave, row8 = at * 8 + lane / 8;
            const uint64_t row = min(m0 + row8, a.m - 1), b = b0 + (lane % 8 ^ (row8 >> 1 & 7));
            load_to_lds(b < a.blocks ? (const void*)(a.x_codes + row * a.blocks + b) : zeros, to_x + at * 1024);
        }
#pragma unroll
        for (int q = 0; q < BN / 8 / kWaves; ++q) {
            // past the end of the depth x is zero, so any finite values do
            const uint32_t at = q * kWaves + wave, row8 = at * 8 + lane / 8;
            const uint64_t row = min(j0 + row8, a.n - 1), b = min(b0 + (lane % 8 ^ (row8 >> 1 & 7)), a.blocks - 1);
            load_to_lds(a.w_codes + row * a.blocks + b, to_w + at * 1024);
        }
    };
    // 16 scale bytes a row: two stages' worth, a lane each
    auto load_scales = [&](uint32_t t, uint8_t* to) {
        const uint64_t b0 = (uint64_t)t * kStepBlocks;
#pragma unroll
        for (int q = 0; q < (BM + BN) / 64 / kWaves; ++q) {
            const uint32_t at = q * kWaves + wave, i = at * 64 + lane;
            const uint8_t* p = at < BM / 64 ? a.x_scales + min(m0 + i, a.m - 1) * a.scale_pitch
                                            : a.w_scales + min(j0 + i - BM, a.n - 1) * a.scale_pitch;
            load_to_lds(p + b0, to + at * 1024);
        }
    };
    // Lane (r, g) multiplies blocks 2 g and 2 g + 1 of its rows.
    const uint32_t c0 = chunk_at(r, 2 * g), c1 = chunk_at(r, 2 * g + 1);
    const uint32_t x_row = wm * FM * 16, w_row = wn * FN * 16;
    auto stage = [&](uint32_t t, const uint8_t* x_now, const uint8_t* w_now, const uint8_t* s_now, uint32_t half) {
        // scale bytes past the row's end may hold anything
        const uint64_t b = (uint64_t)t * kStepBlocks + 2 * g;
        const uint32_t mask = b + 1 < a.blocks ? 0xffff : b < a.blocks ? 0xff : 0;
        uint32_t xs[FM], ws[FN];
#pragma unroll
        for (int m = 0; m < FM; ++m)
            xs[m] = *reinterpret_cast<const uint16_t*>(s_now + ((x_row + m * 16 + r) * 16 + half * 8 + g * 2)) & mask;
#pragma unroll
        for (int n = 0; n < FN; ++n)
            ws[n] = *reinterpret_cast<const uint16_t*>(s_now + ((BM + w_row + n * 16 + r) * 16 + half * 8 + g * 2)) & mask;
        auto step = [&](auto which) {
            constexpr int j = decltype(which)::value;
            u32x4 x[FM];
#pragma unroll
            for (int m = 0; m < FM; ++m) x[m] = *reinterpret_cast<const u32x4*>(x_now + ((x_row + m * 16) * 128 + (j ? c1 : c0)));
#pragma unroll
            for (int n = 0; n < FN; ++n) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(w_now + ((w_row + n * 16) * 128 + (j ? c1 : c0)));
#pragma unroll
                for (int m = 0; m < FM; ++m)
                    acc[n][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(w), fragment(x[m]), acc[n][m], 4, 4,
                                                                                 j, ws[n], j, xs[m]);
            }
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
    };
    // stages t and t + 1 with their scales; those of the next pair into `s_next`
    auto pair = [&](uint32_t t, const uint8_t* s_now, uint8_t* s_next) {
        wait_loads();
        __syncthreads();
        if (t + 1 < t1) load(t + 1, lds_x1, lds_w1);
        if (t + 2 < t1) load_scales(t + 2, s_next);
        stage(t, lds_x0, lds_w0, s_now, 0);
        if (t + 1 >= t1) return;
        wait_loads();
        __syncthreads();
        if (t + 2 < t1) load(t + 2, lds_x0, lds_w0);
        stage(t + 1, lds_x1, lds_w1, s_now, 1);
    };
    if (t0 < t1) {
        load(t0, lds_x0, lds_w0);
        load_scales(t0, lds_s0);
    }
    for (uint32_t t = t0; t < t1; t += 4) {
        pair(t, lds_s0, lds_s1);
        if (t + 2 < t1) pair(t + 2, lds_s1, lds_s0);
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
