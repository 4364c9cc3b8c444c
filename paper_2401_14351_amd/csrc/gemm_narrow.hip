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
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kRowBytes = kNarrowStep / 2;
    // The two stages are variables of their own: the compiler then sees that
    // loads into one do not touch what is read from the other.
    __shared__ __align__(16) uint8_t lds_x0[BM * kRowBytes], lds_x1[BM * kRowBytes];
    __shared__ __align__(16) uint8_t lds_w0[BN * kRowBytes], lds_w1[BN * kRowBytes];
    // scales of two stages: 16 bytes a row, x's rows then w's
    __shared__ __align__(16) uint8_t lds_s0[(BM + BN) * 16], lds_s1[(BM + BN) * 16];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 31, h = lane >> 5;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    const uint32_t wm = wave % WM, wn = wave / WM;
    // splits begin at pairs of stages, which share their scales
    const uint32_t pairs = (a.steps + 1) / 2;
    const uint32_t t0 = (uint64_t)pairs * blockIdx.y / gridDim.y * 2;
    const uint32_t t1 = min((uint32_t)((uint64_t)pairs * (blockIdx.y + 1) / gridDim.y * 2), a.steps);

    f32x16 acc[FN][FM];
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[n][m] = f32x16{};

    // One load holds 8 rows x 8 blocks, and a lane takes the same blocks of each
    // of its rows.
    static_assert(kWaves % 2 == 0, "");
    const uint32_t block = lane % 8 ^ (wave % 2 * 4 + lane / 16);
    const u32x4 *x_at[BM / 8 / kWaves], *w_at[BN / 8 / kWaves];
#pragma unroll
    for (int q = 0; q < BM / 8 / kWaves; ++q)
        x_at[q] = a.x_codes + min(m0 + (q * kWaves + wave) * 8 + lane / 8, a.m - 1) * a.blocks;
#pragma unroll
    for (int q = 0; q < BN / 8 / kWaves; ++q)
        w_at[q] = a.w_codes + min(j0 + (q * kWaves + wave) * 8 + lane / 8, a.n - 1) * a.blocks;
    // 16 scale bytes a row: two stages' worth, a lane each
    static_assert((BM + BN) / 64 == kWaves, "");
    const uint8_t* scales_at = wave < BM / 64 ? a.x_scales + min(m0 + tid, a.m - 1) * a.scale_pitch
                                              : a.w_scales + min(j0 + tid - BM, a.n - 1) * a.scale_pitch;
    auto load = [&](uint32_t t, uint8_t* to_x, uint8_t* to_w) {
        const uint64_t b = (uint64_t)t * kStepBlocks + block, at = min(b, a.blocks - 1);
#pragma unroll
        for (int q = 0; q < BM / 8 / kWaves; ++q) {
            const void* p = x_at[q] + at;
            load_to_lds(b < a.blocks ? p : zeros, to_x + (q * kWaves + wave) * 1024);
        }
        // past the end of the depth x is zero, so any finite values do
#pragma unroll
        for (int q = 0; q < BN / 8 / kWaves; ++q) load_to_lds(w_at[q] + at, to_w + (q * kWaves + wave) * 1024);
    };
    auto load_scales = [&](uint32_t t, uint8_t* to) { load_to_lds(scales_at + (uint64_t)t * kStepBlocks, to + wave * 1024); };

    // Of a stage, lane (r, h) multiplies blocks 4 h .. 4 h + 3 of its rows, one a
    // step; a row's four scale bytes are one register.
    struct Scales {
        uint32_t x[FM], w[FN];
    };
    auto read_scales = [&](uint32_t t, const uint8_t* from) {
        // scale bytes past the row's end may hold anything
        const uint64_t b = (uint64_t)t * kStepBlocks + 4 * h;
        const uint32_t left = b < a.blocks ? (uint32_t)min(a.blocks - b, (uint64_t)4) : 0;
        const uint32_t mask = left == 4 ? ~0u : (1u << left * 8) - 1;
        Scales s;
#pragma unroll
        for (int m = 0; m < FM; ++m)
            s.x[m] = *reinterpret_cast<const uint32_t*>(from + ((wm * FM + m) * 512 + r * 16 + t % 2 * 8 + h * 4)) & mask;
#pragma unroll
        for (int n = 0; n < FN; ++n)
            s.w[n] = *reinterpret_cast<const uint32_t*>(from + (BM * 16 + (wn * FN + n) * 512 + r * 16 + t % 2 * 8 + h * 4)) & mask;
        return s;
    };
    struct Fragments {
        u32x4 x[FM], w[FN];
    };
    const uint32_t chunk = chunk_at(r, 4 * h);
    auto read = [&](const uint8_t* x_now, const uint8_t* w_now, uint32_t s) {
        Fragments f;
        const uint32_t c = chunk ^ s * 16;
#pragma unroll
        for (int n = 0; n < FN; ++n) f.w[n] = *reinterpret_cast<const u32x4*>(w_now + ((wn * FN + n) * 4096 + c));
#pragma unroll
        for (int m = 0; m < FM; ++m) f.x[m] = *reinterpret_cast<const u32x4*>(x_now + ((wm * FM + m) * 4096 + c));
        return f;
    };
    auto multiply = [&](const Fragments& f, const Scales& s, auto which) {
        constexpr int j = decltype(which)::value;
        pin(acc);
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n)
                acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fragment(f.w[n]), fragment(f.x[m]), acc[n][m], 4, 4, j,
                                                                            s.w[n], j, s.x[m]);
        pin(acc);
    };
    // While one step is multiplied the next is read; the next stage's first step
    // past the barrier, where its loads have landed and this stage's buffers are
    // free for the loads of the one after.
    Fragments f0, f1;
    Scales now, next;
    auto stage = [&](uint32_t t, uint8_t* x_now, uint8_t* w_now, const uint8_t* x_next, const uint8_t* w_next, const uint8_t* scales,
                     uint8_t* scales_to) {
        f1 = read(x_now, w_now, 1);
        multiply(f0, now, std::integral_constant<int, 0>());
        f0 = read(x_now, w_now, 2);
        multiply(f1, now, std::integral_constant<int, 1>());
        f1 = read(x_now, w_now, 3);
        multiply(f0, now, std::integral_constant<int, 2>());
        wait_loads();
        __syncthreads();
        if (t + 2 < t1) {
            load(t + 2, x_now, w_now);
            if (scales_to) load_scales(t + 2, scales_to);
        }
        f0 = read(x_next, w_next, 0);
        next = read_scales(t + 1, scales);
        multiply(f1, now, std::integral_constant<int, 3>());
        now = next;
    };
    if (t0 < t1) {
        load(t0, lds_x0, lds_w0);
        load_scales(t0, lds_s0);
        wait_loads();
        __syncthreads();
        if (t0 + 1 < t1) load(t0 + 1, lds_x1, lds_w1);
        f0 = read(lds_x0, lds_w0, 0);
        now = read_scales(t0, lds_s0);
    }
    for (uint32_t t = t0; t < t1; t += 4) {
        stage(t, lds_x0, lds_w0, lds_x1, lds_w1, lds_s0, lds_s1);
        if (t + 1 < t1) {
            stage(t + 1, lds_x1, lds_w1, lds_x0, lds_w0, lds_s1, nullptr);
            if (t + 2 < t1) {
                stage(t + 2, lds_x0, lds_w0, lds_x1, lds_w1, lds_s1, lds_s0);
                if (t + 3 < t1) stage(t + 3, lds_x1, lds_w1, lds_x0, lds_w0, lds_s0, nullptr);
            }
        }
    }
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 32, j0 + wn * FN * 32, out);
}

}  // namespace

int32_t launch_narrow(const NarrowArgs& a, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, (narrow_product<256, 256, 2, 4, T><<<grid, 512, 0, stream>>>(a, static_cast<T*>(out))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
