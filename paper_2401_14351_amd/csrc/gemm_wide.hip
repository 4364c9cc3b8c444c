// gfx950 kernels of products with an MX FP4 weight and an x of 16 or 32 bits.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStep = kWideStep;

template <int BM, int BN, int WM, int WN, typename T>
__global__ __launch_bounds__(WM* WN * 64) void wide_product(WideArgs a, T* out) {
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kXLoads = BM / 8 / kWaves, kWLoads = BN / 16 / kWaves, kScaleWaves = BN / 64;
    constexpr int kXBytes = BM * kStep * 2, kWBytes = BN * 64, kScaleBytes = BN * 4;
    static_assert(kScaleWaves <= kWaves, "");
    // The stages are variables of their own: the compiler then sees that loads
    // into one do not touch what is read from another.
    __shared__ __align__(16) uint8_t lds_x0[kXBytes], lds_x1[kXBytes];
    // W and its scales, of two stages
    __shared__ __align__(16) uint8_t lds_w0[kWBytes + kScaleBytes], lds_w1[kWBytes + kScaleBytes];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 31, h = lane >> 5;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    // a part's steps are even: stages go in pairs that share a piece of W
    const uint32_t pairs = a.steps / 2 * a.parts;
    const uint32_t t0 = (uint64_t)pairs * blockIdx.y / gridDim.y * 2, t1 = (uint64_t)pairs * (blockIdx.y + 1) / gridDim.y * 2;
    const uint32_t wm = wave % WM, wn = wave / WM;

    f32x16 acc[FN][FM];
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[n][m] = f32x16{};

    // x by loads straight to LDS: one load holds 8 rows x 64 of the depth, and
    // a lane takes the same columns of each of its rows
    static_assert(kWaves % 2 == 0, "");
    const uint32_t x_col = (lane % 8 ^ (wave % 2 * 4 + lane / 16)) * 8;
    const __bf16* x_at[kXLoads];
#pragma unroll
    for (int q = 0; q < kXLoads; ++q) x_at[q] = a.x + min(m0 + (q * kWaves + wave) * 8 + lane / 8, a.m - 1) * a.x_stride + x_col;
    auto load_x = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint32_t part = t / a.steps;
        const uint64_t d = (uint64_t)(t - part * a.steps) * kStep, at = part * a.part_stride + d;
        const bool inside = d + x_col < a.depth;
#pragma unroll
        for (int q = 0; q < kXLoads; ++q) {
            const void* p = x_at[q] + at;
            load_to_lds(inside ? p : zeros, to + (q * kWaves + wave) * 1024);
        }
    };
    // W's codes likewise, one load 16 rows x 128 of the depth, and four scale
    // bytes a row.  Past the end of the depth x is zero, so any codes do.
    const uint32_t w_block = lane % 4 ^ lane / 16;
    const u32x4* w_at[kWLoads];
#pragma unroll
    for (int q = 0; q < kWLoads; ++q) w_at[q] = a.w_codes + min(j0 + (q * kWaves + wave) * 16 + lane / 4, a.w_rows - 1) * a.w_blocks;
    const uint8_t* scales_at = a.w_scales + min(j0 + (wave % kScaleWaves) * 64 + lane, a.w_rows - 1) * a.w_scale_pitch;
    auto load_w = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint64_t b0 = (uint64_t)(t % a.steps) * 2, b = min(b0 + w_block, a.w_blocks - 1);
#pragma unroll
        for (int q = 0; q < kWLoads; ++q) load_to_lds(w_at[q] + b, to + (q * kWaves + wave) * 1024);
        if (wave < kScaleWaves) load_word_to_lds(scales_at + b0, to + (kWBytes + wave * 256));
    };

    // Of a stage, lane (r, h) has 32 of the depth of its rows: the block of W
    // that it expands as it goes, eight codes a step.
    struct Weight {
        u32x4 codes[FN];
        float scale[FN];
    };
    const uint32_t w_chunk = short_chunk_at(r, h);
    auto read_w = [&](uint32_t t, const uint8_t* from, uint32_t odd) SLLM_INLINE {
        const bool inside = (uint64_t)(t % a.steps) * 2 + h < a.w_blocks;  // scale bytes past the row's end may hold anything
        Weight w;
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            w.codes[n] = *reinterpret_cast<const u32x4*>(from + ((wn * FN + n) * 2048 + (w_chunk ^ odd * 32)));
            const uint8_t s = from[kWBytes + ((wn * FN + n) * 128 + r * 4 + h + odd * 2)];
            w.scale[n] = mx_scale(inside ? s : 0);
        }
        return w;
    };

    struct Fragments {
        bf16x8 x[FM], w[FN];
    };
    // Step s of a stage is, in lane (r, h), eight of the depth from 32 h + 8 s.
    const uint32_t chunk = chunk_at(r, 4 * h);
    auto read = [&](const uint8_t* from, const Weight& w, auto which) SLLM_INLINE {
        constexpr int s = decltype(which)::value;
        Fragments f;
        const uint32_t c = chunk ^ s * 16;
#pragma unroll
        for (int m = 0; m < FM; ++m) f.x[m] = *reinterpret_cast<const bf16x8*>(from + ((wm * FM + m) * 4096 + c));
#pragma unroll
        for (int n = 0; n < FN; ++n) f.w[n] = __builtin_bit_cast(bf16x8, expand8(w.codes[n][s], w.scale[n]));
        return f;
    };
    auto multiply = [&](const Fragments& f) SLLM_INLINE {
        pin(acc);
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.w[n], f.x[m], acc[n][m], 0, 0, 0);
        pin(acc);
    };
    // While one step is multiplied the next is read; the next stage's first step
    // past the barrier, where its loads have landed and this stage's buffers are
    // free for the loads of the one after.
    typedef std::integral_constant<int, 0> S0;
    typedef std::integral_constant<int, 1> S1;
    typedef std::integral_constant<int, 2> S2;
    typedef std::integral_constant<int, 3> S3;
    Fragments f0, f1;
    Weight now;
    auto stage = [&](uint32_t t, uint8_t* x_now, const uint8_t* x_next, const uint8_t* w_next, uint32_t odd_next, auto load_more) SLLM_INLINE {
        f1 = read(x_now, now, S1());
        multiply(f0);
        f0 = read(x_now, now, S2());
        multiply(f1);
        f1 = read(x_now, now, S3());
        multiply(f0);
        wait_but_loads<0>();
        barrier();
        now = read_w(t + 1, w_next, odd_next);
        if (t + 2 < t1) load_x(t + 2, x_now);
        load_more();
        f0 = read(x_next, now, S0());
        multiply(f1);
    };
    // a pair of stages whose W is in w_now; the pair after the next goes there
    auto pair = [&](uint32_t t, uint8_t* w_now, const uint8_t* w_next) SLLM_INLINE {
        stage(t, lds_x0, lds_x1, w_now, 1, []() SLLM_INLINE {});
        stage(t + 1, lds_x1, lds_x0, w_next, 0, [&]() SLLM_INLINE {
            if (t + 4 < t1) load_w(t + 4, w_now);
        });
    };
    if (t0 < t1) {
        load_x(t0, lds_x0);
        load_w(t0, lds_w0);
        wait_but_loads<0>();
        barrier();
        load_x(t0 + 1, lds_x1);
        if (t0 + 2 < t1) load_w(t0 + 2, lds_w1);
        now = read_w(t0, lds_w0, 0);
        f0 = read(lds_x0, now, S0());
        for (uint32_t t = t0; t < t1; t += 4) {
            pair(t, lds_w0, lds_w1);
            if (t + 2 < t1) pair(t + 2, lds_w1, lds_w0);
        }
    }

    __syncthreads();  // the last stage's reads are done
    // the output goes through a buffer of x
    static_assert(kXBytes >= kWaves * kTurnBytes, "");
    uint8_t* const turn = lds_x0 + wave * kTurnBytes;
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 32, j0 + wn * FN * 32, out, turn);
}

}  // namespace

int32_t launch_wide(const WideArgs& a, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, (wide_product<256, 256, 2, 4, T><<<grid, 512, 0, stream>>>(a, static_cast<T*>(out))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
