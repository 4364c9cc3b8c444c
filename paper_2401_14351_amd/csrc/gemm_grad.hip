// gfx950 kernel of dy times an MX FP4 weight: the gradient by a product's input.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStep = kWideStep;

template <int BM, int BN, int WM, int WN, typename T>
__global__ __launch_bounds__(WM* WN * 64) void grad_product(WideArgs a, T* out) {
    constexpr int kThreads = WM * WN * 64, kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kLoads = BM / 8 / kWaves;               // loads of x a wave issues a stage
    constexpr int kBlocks = BN * kStep / 32 / kThreads;   // blocks of W a lane expands a stage
    constexpr int kPitch = BN * 2 + 32;                   // bytes of a row of W's tile in LDS
    constexpr int kXBytes = BM * kStep * 2, kWBytes = kStep * kPitch;
    // The two stages are variables of their own: the compiler then sees that
    // loads into one do not touch what is read from the other.
    __shared__ __align__(16) uint8_t lds_x0[kXBytes], lds_x1[kXBytes];
    __shared__ __align__(16) uint8_t lds_w0[kWBytes], lds_w1[kWBytes];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 31, h = lane >> 5;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    const uint32_t steps = a.steps * a.parts;
    const uint32_t t0 = (uint64_t)steps * blockIdx.y / gridDim.y, t1 = (uint64_t)steps * (blockIdx.y + 1) / gridDim.y;
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
    const __bf16* x_at[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) x_at[q] = a.x + min(m0 + (q * kWaves + wave) * 8 + lane / 8, a.m - 1) * a.x_stride + x_col;
    auto load_x = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint32_t part = t / a.steps;
        const uint64_t d = (uint64_t)(t - part * a.steps) * kStep, at = part * a.part_stride + d;
        const bool inside = d + x_col < a.depth;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const void* p = x_at[q] + at;
            load_to_lds(inside ? p : zeros, to + (q * kWaves + wave) * 1024);
        }
    };
    // The blocks a lane expands, of two stages: a row's are neighbours then.
    // Past the end of the depth x is zero, so any codes do under a finite scale.
    u32x4 codes[2][kBlocks];
    uint32_t scales[2][kBlocks];
    const uint32_t w_row = tid / (BN / 32), w_block = tid % (BN / 32);
    auto load_w = [&](uint32_t t, int to) SLLM_INLINE {
        const uint64_t s = t % a.steps;
#pragma unroll
        for (int q = 0; q < kBlocks; ++q) {
            const uint64_t row_at = min(s * kStep + w_row + q * (kThreads / (BN / 32)), a.w_rows - 1);
            const uint64_t b_at = min(j0 / 32 + w_block, a.w_blocks - 1);
            codes[to][q] = a.w_codes[row_at * a.w_blocks + b_at];
            scales[to][q] = a.w_scales[row_at * a.w_scale_pitch + b_at];
        }
    };
    // W's tile in LDS: rows of the depth by the tile's columns, whose order
    // changes from block to block so that a wave's stores reach all banks.
    auto store_w = [&](uint32_t t, int from, uint8_t* to) SLLM_INLINE {
        const uint64_t s = t % a.steps;
#pragma unroll
        for (int q = 0; q < kBlocks; ++q) {
            const bool inside = s * kStep + w_row + q * (kThreads / (BN / 32)) < a.w_rows;
            u32x4 v[4];
            expand(codes[from][q], inside ? scales[from][q] : 0, v);
            const uint32_t i = q * kThreads + tid;
#pragma unroll
            for (uint32_t w = 0; w < 4; ++w) {
                const uint32_t at = i / (BN / 32) * kPitch + w_block * 64 + (w ^ (i & 3)) * 16;
                *reinterpret_cast<u32x4*>(to + at) = v[w];
            }
        }
    };

    struct Fragments {
        bf16x8 x[FM], w[FN];
    };
    // Step s of a stage is, in lane (r, h), eight of the depth from 32 h + 8 s.
    const uint32_t chunk = chunk_at(r, 4 * h);
    auto read = [&](const uint8_t* x_now, const uint8_t* w_now, uint32_t s) SLLM_INLINE {
        Fragments f;
        const uint32_t c = chunk ^ s * 16;
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            // Four rows of the tile and 16 columns a read and 16 lanes,
            // transposed: a lane gets a column.
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const uint32_t b = wn * FN + n, l = lane & 15;
            const uint32_t piece = ((lane >> 4 & 1) * 2 + (l >> 1 & 1)) ^ (b & 3);
            const uint32_t at = (32 * h + 8 * s + (l >> 2)) * kPitch + b * 64 + piece * 16 + (l & 1) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(w_now + at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(w_now + (at + 4 * kPitch)));
            f.w[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
        for (int m = 0; m < FM; ++m) f.x[m] = *reinterpret_cast<const bf16x8*>(x_now + ((wm * FM + m) * 4096 + c));
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
    Fragments f0, f1;
    auto stage = [&](uint32_t t, int parity, uint8_t* x_now, const uint8_t* w_now, const uint8_t* x_next, uint8_t* w_next) SLLM_INLINE {
        f1 = read(x_now, w_now, 1);
        multiply(f0);
        f0 = read(x_now, w_now, 2);
        multiply(f1);
        f1 = read(x_now, w_now, 3);
        if (t + 1 < t1) store_w(t + 1, parity ^ 1, w_next);
        multiply(f0);
        wait_but_loads<0>();
        barrier();
        if (t + 2 < t1) {
            load_x(t + 2, x_now);
            if (parity == 0) {
                load_w(t + 2, 0);
                load_w(t + 3, 1);
            }
        }
        f0 = read(x_next, w_next, 0);
        multiply(f1);
    };
    if (t0 < t1) {
        load_x(t0, lds_x0);
        load_w(t0, 0);
        load_w(t0 + 1, 1);
        store_w(t0, 0, lds_w0);
        wait_but_loads<0>();
        barrier();
        if (t0 + 1 < t1) load_x(t0 + 1, lds_x1);
        f0 = read(lds_x0, lds_w0, 0);
    }
    for (uint32_t t = t0; t < t1; t += 2) {
        stage(t, 0, lds_x0, lds_w0, lds_x1, lds_w1);
        if (t + 1 < t1) stage(t + 1, 1, lds_x1, lds_w1, lds_x0, lds_w0);
    }

    __syncthreads();  // the last stage's reads are done
    // the output goes through a buffer of x
    static_assert(kXBytes >= kWaves * kTurnBytes, "");
    uint8_t* const turn = lds_x0 + wave * kTurnBytes;
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 32, j0 + wn * FN * 32, out, turn);
}

}  // namespace

int32_t launch_grad(const WideArgs& a, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, (grad_product<256, 256, 2, 4, T><<<grid, 512, 0, stream>>>(a, static_cast<T*>(out))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
