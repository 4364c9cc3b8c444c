// gfx950 kernel of products with both sides in MX FP4.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStepBlocks = kNarrowStep / kMxBlock;
constexpr uint32_t kStageBlocks = 4;  // of a stage: 64 bytes a row

// out[m][n] = sum over k of x[m][k] W[n][k], both in four bits, in 32 bits: the
// scaled matrix instruction takes codes and scales as they are stored.  4096 x 8192 by
// 28672 takes 500 to 540 us, 3.6 to 3.85 PF/s: the matrix cores are busy 48 % of the
// cycles at 1.85 to 1.9 GHz, alone 6.8 to 7.3 PF/s at 1.63 to 1.94.  LDS is in use 38 % of
// the cycles, over a third of that conflicts, whose cause, the fragments' reads or those of
// the scales, has not been separated.
//
// A stage of 128 of the depth is 64 bytes a row: four of them are in flight, loaded
// straight to LDS, and waited for by their number, not all together.  512 of the
// depth share a load of scales, 16 bytes a row.
template <int BM, int BN, int WM, int WN, typename T>
__global__ __launch_bounds__(WM* WN * 64, 2) void narrow_product(NarrowArgs a, T* out) {
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    // The stages in flight are variables of their own: the compiler then sees
    // that loads into one do not touch what is read from another.
    constexpr int kStageBytes = (BM + BN) * 64;
    __shared__ __align__(16) uint8_t b0[kStageBytes], b1[kStageBytes], b2[kStageBytes], b3[kStageBytes];
    // scales of four stages: 16 bytes a row, x's rows then w's
    __shared__ __align__(16) uint8_t s0[(BM + BN) * 16], s1[(BM + BN) * 16];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 31, h = lane >> 5;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    const uint32_t wm = wave % WM, wn = wave / WM;
    const uint32_t t0 = (uint64_t)a.steps * blockIdx.y / gridDim.y, t1 = (uint64_t)a.steps * (blockIdx.y + 1) / gridDim.y;

    f32x16 acc[FN][FM];
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[n][m] = f32x16{};

    // One load holds 16 rows x 4 blocks, and a lane takes the same block of each
    // of its rows.
    constexpr int kXLoads = BM / 16 / kWaves, kWLoads = BN / 16 / kWaves;
    const uint32_t block = lane % 4 ^ lane / 16;
    const u32x4 *x_at[kXLoads], *w_at[kWLoads];
#pragma unroll
    for (int q = 0; q < kXLoads; ++q) x_at[q] = a.x_codes + min(m0 + (q * kWaves + wave) * 16 + lane / 4, a.m - 1) * a.blocks;
#pragma unroll
    for (int q = 0; q < kWLoads; ++q) w_at[q] = a.w_codes + min(j0 + (q * kWaves + wave) * 16 + lane / 4, a.n - 1) * a.blocks;
    // 16 scale bytes a row: four stages' worth, a lane each
    constexpr int kScaleLoads = (BM + BN) / 64 / kWaves;
    const uint8_t* scales_at[kScaleLoads];
#pragma unroll
    for (int q = 0; q < kScaleLoads; ++q) {
        const uint32_t at = q * kWaves + wave, i = at * 64 + lane;
        scales_at[q] = at < BM / 64 ? a.x_scales + min(m0 + i, a.m - 1) * a.scale_pitch
                                    : a.w_scales + min(j0 + i - BM, a.n - 1) * a.scale_pitch;
    }
    // Stages are counted in blocks of the depth.  Every stage loads, those past
    // the end too, so that the loads to wait for can be told by their number.
    constexpr int kLoads = kXLoads + kWLoads;
    auto load = [&](uint64_t at, uint8_t* to) SLLM_INLINE {
        const uint64_t b = at + block, inside = min(b, a.blocks - 1);
#pragma unroll
        for (int q = 0; q < kXLoads; ++q) {
            const void* p = x_at[q] + inside;
            load_to_lds(b < a.blocks ? p : zeros, to, (q * kWaves + wave) * 1024);
        }
        // past the end of the depth x is zero, so any finite values do
#pragma unroll
        for (int q = 0; q < kWLoads; ++q) load_to_lds(w_at[q] + inside, to, BM * 64 + (q * kWaves + wave) * 1024);
    };
    auto load_scales = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint64_t b = min((uint64_t)t * kStepBlocks, a.scale_pitch - kStepBlocks);
#pragma unroll
        for (int q = 0; q < kScaleLoads; ++q) load_to_lds(scales_at[q] + b, to, (q * kWaves + wave) * 1024);
    };

    // Of a stage, lane (r, h) multiplies blocks 2 h and 2 h + 1 of its rows, one a
    // step; a row's two scale bytes are one register.
    // (Filled through a reference: a returned structure makes its reads' alias
    // information useless, and they wait for every load under way.)
    struct Scales {
        uint32_t x[FM], w[FN];
    };
    const uint32_t xs_from = opaque(wm * FM * 512 + r * 16 + h * 2), ws_from = opaque((BM + wn * FN * 32 + r) * 16 + h * 2);
    auto read_scales = [&](Scales& s, uint64_t at, const uint8_t* from, uint32_t stage) SLLM_INLINE {
        // scale bytes past the row's end may hold anything
        const uint64_t b = at + 2 * h;
        const uint32_t mask = b + 1 < a.blocks ? 0xffff : b < a.blocks ? 0xff : 0;
#pragma unroll
        for (int m = 0; m < FM; ++m)
            s.x[m] = lds_read<uint16_t>(from, xs_from + m * 512 + stage * 4) & mask;
#pragma unroll
        for (int n = 0; n < FN; ++n)
            s.w[n] = lds_read<uint16_t>(from, ws_from + n * 512 + stage * 4) & mask;
    };
    struct Fragments {
        u32x4 x[FM], w[FN];
    };
    const uint32_t x_from = opaque(wm * FM * 2048 + short_chunk_at(r, 2 * h));
    const uint32_t w_from = opaque(BM * 64 + wn * FN * 2048 + short_chunk_at(r, 2 * h));
    auto read = [&](Fragments& f, const uint8_t* from, uint32_t s) SLLM_INLINE {
#pragma unroll
        for (int n = 0; n < FN; ++n) f.w[n] = lds_read<u32x4>(from, (w_from ^ s * 16) + n * 2048);
#pragma unroll
        for (int m = 0; m < FM; ++m) f.x[m] = lds_read<u32x4>(from, (x_from ^ s * 16) + m * 2048);
    };
    auto multiply = [&](const Fragments& f, const Scales& s, auto which) SLLM_INLINE {
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
    // A ring of four stages, three of them in flight.  While one step is
    // multiplied the next is read; the next stage's first step past the barrier,
    // where its loads have landed.  The buffer of the stage before is free from
    // its barrier on and takes the loads of the third stage ahead.
    Fragments f0, f1;
    Scales now;
    auto stage = [&](uint64_t at, const uint8_t* here, const uint8_t* next_one, uint8_t* last, const uint8_t* scales,
                     uint32_t next_stage, auto more) SLLM_INLINE {
        read(f1, here, 1);
        load(at + 3 * kStageBlocks, last);
        more();
        multiply(f0, now, std::integral_constant<int, 0>());
        wait_but_loads<2 * kLoads>();  // younger than the next stage's: those of the two after it
        barrier();
        read(f0, next_one, 0);
        Scales next;
        read_scales(next, at + kStageBlocks, scales, next_stage);
        multiply(f1, now, std::integral_constant<int, 1>());
        now = next;
    };
    auto four_stages = [&](uint32_t t, uint8_t* s_now, uint8_t* s_next) SLLM_INLINE {
        const uint64_t at = (uint64_t)t * kStepBlocks;
        const auto none = []() SLLM_INLINE {};
        stage(at, b0, b1, b3, s_now, 1, [&]() SLLM_INLINE { load_scales(t + 1, s_next); });
        stage(at + 4, b1, b2, b0, s_now, 2, none);
        stage(at + 8, b2, b3, b1, s_now, 3, none);
        stage(at + 12, b3, b0, b2, s_next, 0, none);
    };
    if (t0 < t1) {
        const uint64_t at = (uint64_t)t0 * kStepBlocks;
        load_scales(t0, s0);
        load(at, b0);
        load(at + 4, b1);
        load(at + 8, b2);
        wait_but_loads<2 * kLoads>();
        barrier();
        read(f0, b0, 0);
        read_scales(now, at, s0, 0);
        for (uint32_t t = t0; t < t1; t += 2) {
            four_stages(t, s0, s1);
            if (t + 1 < t1) four_stages(t + 1, s1, s0);
        }
        wait_but_loads<0>();
        barrier();
    }
    // the output goes through a stage's buffer
    static_assert(kStageBytes >= kWaves * kTurnBytes, "");
    uint8_t* const turn = b0 + wave * kTurnBytes;
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 32, j0 + wn * FN * 32, out, turn);
}

}  // namespace

int32_t launch_narrow(const NarrowArgs& a, uint32_t tile, uint32_t splits, void* out, uint32_t out_dtype,
                    hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, {
        T* to = static_cast<T*>(out);
        if (tile == kLargeTile)
            narrow_product<kLargeTile, kLargeTile, 2, 4, T><<<grid, 512, 0, stream>>>(a, to);
        else
            narrow_product<kSmallTile, kSmallTile, 2, 2, T><<<grid, 256, 0, stream>>>(a, to);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
