// gfx950 kernels of products with an MX FP4 weight and an x of 16 or 32 bits.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStep = kWideStep;

template <bool Grad, int BM, int BN, int WM, int WN>
struct Wide {
    static constexpr int kThreads = WM * WN * 64, kWaves = WM * WN;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;     // fragments of a wave
    static constexpr int kPitch = BN * 2 + 32;                     // bytes of a row of W's tile in LDS (Grad)
    static constexpr int kABytes = BM * kStep * 2;
    static constexpr int kBBytes = Grad ? kStep * kPitch : BN * kStep * 2;
    static constexpr int kBlocks = BN * kStep / 32 / kThreads;     // blocks of W a lane expands a stage
    static constexpr int kLoads = BM / 8 / kWaves;                 // loads of x a wave issues a stage
};

template <bool Grad, int BM, int BN, int WM, int WN, typename T>
__global__ __launch_bounds__(WM* WN * 64) void wide_product(WideArgs a, T* out) {
    using G = Wide<Grad, BM, BN, WM, WN>;
    // The two stages are variables of their own: the compiler then sees that
    // loads into one do not touch what is read from the other.
    __shared__ __align__(16) uint8_t lds_a0[G::kABytes], lds_a1[G::kABytes];
    __shared__ __align__(16) uint8_t lds_b0[G::kBBytes], lds_b1[G::kBBytes];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 15, g = lane >> 4;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    const uint32_t steps = a.steps * a.parts;
    const uint32_t t0 = (uint64_t)steps * blockIdx.y / gridDim.y, t1 = (uint64_t)steps * (blockIdx.y + 1) / gridDim.y;

    f32x4 acc[G::FN][G::FM];
#pragma unroll
    for (int n = 0; n < G::FN; ++n)
#pragma unroll
        for (int m = 0; m < G::FM; ++m) acc[n][m] = f32x4{0, 0, 0, 0};

    // x by loads straight to LDS: one load holds 8 rows x 64 of the depth, and
    // a lane takes the same columns of each of its rows
    static_assert(G::kWaves % 2 == 0, "");
    const uint32_t x_col = (lane % 8 ^ (wave % 2 * 4 + lane / 16)) * 8;
    const __bf16* x_at[G::kLoads];
#pragma unroll
    for (int q = 0; q < G::kLoads; ++q)
        x_at[q] = a.x + min(m0 + (q * G::kWaves + wave) * 8 + lane / 8, a.m - 1) * a.x_stride + x_col;
    auto load_x = [&](uint32_t t, uint8_t* to) {
        const uint32_t part = t / a.steps;
        const uint64_t d = (uint64_t)(t - part * a.steps) * kStep, at = part * a.part_stride + d;
        const bool inside = d + x_col < a.depth;
#pragma unroll
        for (int q = 0; q < G::kLoads; ++q) {
            const void* p = x_at[q] + at;
            load_to_lds(inside ? p : zeros, to + (q * G::kWaves + wave) * 1024);
        }
    };
    // The blocks a lane expands, of two stages: a row's are neighbours then.
    // Past the end of the depth x is zero, so any codes do under a finite scale.
    u32x4 codes[2][G::kBlocks];
    uint32_t scales[2][G::kBlocks];
    const uint32_t w_in = Grad ? tid / (BN / 32) : tid % 2;  // this lane's place in a stage's depth: row or block
    auto load_w = [&](uint32_t t, int to) {
        const uint64_t s = t % a.steps;
#pragma unroll
        for (int q = 0; q < G::kBlocks; ++q) {
            const uint64_t row = Grad ? s * kStep + w_in + q * (G::kThreads / (BN / 32)) : j0 + (q * G::kThreads + tid) / 2;
            const uint64_t b = Grad ? j0 / 32 + tid % (BN / 32) : s * 2 + w_in;
            const uint64_t row_at = min(row, a.w_rows - 1), b_at = min(b, a.w_blocks - 1);
            codes[to][q] = a.w_codes[row_at * a.w_blocks + b_at];
            scales[to][q] = a.w_scales[row_at * a.w_scale_pitch + b_at];
        }
    };
    auto store_w = [&](uint32_t t, int from, uint8_t* to) {
        const uint64_t s = t % a.steps;
#pragma unroll
        for (int q = 0; q < G::kBlocks; ++q) {
            const bool inside = Grad ? s * kStep + w_in + q * (G::kThreads / (BN / 32)) < a.w_rows : s * 2 + w_in < a.w_blocks;
            u32x4 v[4];
            expand(codes[from][q], inside ? scales[from][q] : 0, v);
            const uint32_t i = q * G::kThreads + tid;
            if constexpr (Grad) {
                const uint32_t row = i / (BN / 32), b = i % (BN / 32);
                uint8_t* p = to + row * G::kPitch + b * 64;
#pragma unroll
                for (uint32_t w = 0; w < 4; ++w) *reinterpret_cast<u32x4*>(p + (w ^ (b & 3)) * 16) = v[w];
            } else {
                const uint32_t row = i / 2, b = i % 2;
                uint8_t* p = to + row / 16 * 2048 + b * 512 + row % 16 * 16;
#pragma unroll
                for (uint32_t w = 0; w < 4; ++w) *reinterpret_cast<u32x4*>(p + w % 2 * 1024 + w / 2 * 256) = v[w];
            }
        }
    };

    const uint32_t wm = wave % WM, wn = wave / WM;
    const uint32_t c0 = chunk_at(r, 2 * g), c1 = chunk_at(r, 2 * g + 1);
    auto stage = [&](const uint8_t* a_now, const uint8_t* b_now) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            bf16x8 x[G::FM], w[G::FN];
#pragma unroll
            for (int m = 0; m < G::FM; ++m) x[m] = *reinterpret_cast<const bf16x8*>(a_now + ((wm * G::FM + m) * 2048 + (j ? c1 : c0)));
#pragma unroll
            for (int n = 0; n < G::FN; ++n) {
                if constexpr (Grad) {
                    // four rows of the tile and 16 columns a read, transposed: lane r gets column r
                    const uint32_t f = wn * G::FN + n, b = f >> 1;
                    const uint32_t piece = (2 * (f & 1) + (r >> 1 & 1)) ^ (b & 3);
                    const uint8_t* p = b_now + (16 * g + 8 * j + (r >> 2)) * G::kPitch + b * 64 + piece * 16 + (r & 1) * 8;
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * G::kPitch));
                    w[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                } else {
                    w[n] = *reinterpret_cast<const bf16x8*>(b_now + (wn * G::FN * 2048 + lane * 16 + n * 2048 + j * 1024));
                }
            }
#pragma unroll
            for (int n = 0; n < G::FN; ++n)
#pragma unroll
                for (int m = 0; m < G::FM; ++m)
                    acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[n], x[m], acc[n][m], 0, 0, 0);
        }
    };
    if (t0 < t1) {
        load_x(t0, lds_a0);
        load_w(t0, 0);
        load_w(t0 + 1, 1);
        store_w(t0, 0, lds_b0);
    }
    for (uint32_t t = t0; t < t1; t += 2) {
        wait_loads();
        __syncthreads();
        if (t + 1 < t1) load_x(t + 1, lds_a1);
        stage(lds_a0, lds_b0);
        if (t + 1 < t1) {
            store_w(t + 1, 1, lds_b1);
            wait_loads();
            __syncthreads();
            if (t + 2 < t1) {
                load_x(t + 2, lds_a0);
                load_w(t + 2, 0);
                load_w(t + 3, 1);
            }
            stage(lds_a1, lds_b1);
            if (t + 2 < t1) store_w(t + 2, 0, lds_b0);
        }
    }

    store_tile<G::FM, G::FN>(acc, a.out_args, m0 + wm * G::FM * 16, j0 + wn * G::FN * 16, out);
}

}  // namespace

template <bool Grad>
int32_t launch_wide(const WideArgs& a, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, (wide_product<Grad, 256, 256, 2, 4, T><<<grid, 512, 0, stream>>>(a, static_cast<T*>(out))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}
template int32_t launch_wide<false>(const WideArgs&, uint32_t, void*, uint32_t, hipStream_t);
template int32_t launch_wide<true>(const WideArgs&, uint32_t, void*, uint32_t, hipStream_t);

}  // namespace sllm
