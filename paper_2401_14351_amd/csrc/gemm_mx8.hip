// gfx950 kernel of products of an x in MX FP8 with a weight in MX FP4.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kGroupBlocks = kNarrowStep / kMxBlock;  // whose scales are loaded together
constexpr uint32_t kStageBlocks = 2;

// Where chunk c of two of row r lies, rows of 32 bytes: 16 rows read in one column of
// chunks are in all banks once.
__device__ __forceinline__ uint32_t pair_at(uint32_t r, uint32_t c) { return r * 32 + (c ^ (r >> 3 & 1)) * 16; }

// out[m][n] = sum over k of x[m][k] W[n][k], x in eight bits and W in four, in 32 bits: the
// scaled matrix instruction takes both, and their scales, as they are stored.
//
// A stage of 64 of the depth is 64 bytes a row of x and 32 of W: four of them are in flight,
// loaded straight to LDS, and waited for by their number.  Bound by the matrix cores, whose
// clock falls under it, and their waits: 4096 x 8192 by 28672 829 to 875 us, 2.2 to 2.3 PF/s (the
// library's product of 8192 cubed, both sides in eight bits, 2.7), busy 55 % of the cycles.  512 of the depth share a load
// of scales, 16 bytes a row.  Of a stage, a lane (r, h) of the instruction holds, in eight
// bits, elements 16 h to 16 h + 15 of both blocks, and in four all of block h, and gives
// the scale of block h.
template <int BM, int BN, int WM, int WN, typename T>
__global__ __launch_bounds__(WM* WN * 64, 2) void mx8_product(NarrowArgs a, T* out) {
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kStageBytes = BM * 64 + BN * 32;
    // variables of their own: the compiler then sees that loads into one do not touch
    // what is read from another
    __shared__ __align__(16) uint8_t b0[kStageBytes], b1[kStageBytes], b2[kStageBytes], b3[kStageBytes];
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

    // A load holds 16 rows x 4 chunks of x, or 32 rows x 2 of W; a lane takes the same chunk
    // of each of its rows.
    constexpr int kXLoads = BM / 16 / kWaves, kWLoads = BN / 32 / kWaves, kLoads = kXLoads + kWLoads;
    static_assert(kXLoads * 16 * kWaves == BM && kWLoads * 32 * kWaves == BN, "");
    const uint32_t x_chunk = lane % 4 ^ lane / 16, w_chunk = lane % 2 ^ lane / 16 % 2;
    const u32x4 *x_at[kXLoads], *w_at[kWLoads];
#pragma unroll
    for (int q = 0; q < kXLoads; ++q) x_at[q] = a.x_codes + min(m0 + (q * kWaves + wave) * 16 + lane / 4, a.m - 1) * a.blocks * 2;
#pragma unroll
    for (int q = 0; q < kWLoads; ++q) w_at[q] = a.w_codes + min(j0 + (q * kWaves + wave) * 32 + lane / 2, a.n - 1) * a.blocks;
    constexpr int kScaleLoads = (BM + BN) / 64 / kWaves;
    const uint8_t* scales_at[kScaleLoads];
#pragma unroll
    for (int q = 0; q < kScaleLoads; ++q) {
        const uint32_t at = q * kWaves + wave, i = at * 64 + lane;
        scales_at[q] = at < BM / 64 ? a.x_scales + min(m0 + i, a.m - 1) * a.scale_pitch
                                    : a.w_scales + min(j0 + i - BM, a.n - 1) * a.scale_pitch;
    }
    // Stages are counted in blocks of the depth.  Every stage loads, those past the end too,
    // so that the loads to wait for can be told by their number.
    auto load = [&](uint64_t at, uint8_t* to) SLLM_INLINE {
        const uint64_t bx = at + x_chunk / 2, bw = at + w_chunk;
#pragma unroll
        for (int q = 0; q < kXLoads; ++q) {
            const void* p = x_at[q] + min(bx, a.blocks - 1) * 2 + x_chunk % 2;
            load_to_lds(bx < a.blocks ? p : zeros, to, (q * kWaves + wave) * 1024);
        }
        // past the end of the depth x is zero, so any finite values do
#pragma unroll
        for (int q = 0; q < kWLoads; ++q) load_to_lds(w_at[q] + min(bw, a.blocks - 1), to, BM * 64 + (q * kWaves + wave) * 1024);
    };
    auto load_scales = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint64_t b = min((uint64_t)t * kGroupBlocks, a.scale_pitch - kGroupBlocks);
#pragma unroll
        for (int q = 0; q < kScaleLoads; ++q) load_to_lds(scales_at[q] + b, to, (q * kWaves + wave) * 1024);
    };

    // Scales of four stages, two words a row: of stage i block h's is byte 2 (i % 2) of word i / 2.
    struct Scales {
        u32x2 x[FM], w[FN];
    };
    const uint32_t xs_from = opaque((wm * FM * 32 + r) * 16), ws_from = opaque((BM + wn * FN * 32 + r) * 16);
    auto read_scales = [&](Scales& s, uint64_t at, const uint8_t* from, uint32_t half) SLLM_INLINE {
        u32x2 mask;  // scale bytes past the row's end may hold anything
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t b = at + half * 8 + 4 * i + h;
            mask[i] = b + 2 < a.blocks ? 0xff00ff : b < a.blocks ? 0xff : 0;
        }
#pragma unroll
        for (int m = 0; m < FM; ++m) s.x[m] = lds_read<u32x2>(from, xs_from + m * 512 + half * 8) >> 8 * h & mask;
#pragma unroll
        for (int n = 0; n < FN; ++n) s.w[n] = lds_read<u32x2>(from, ws_from + n * 512 + half * 8) >> 8 * h & mask;
    };
    struct Fragments {
        u32x4 x[FM][2], w[FN];
    };
    const uint32_t x_from = opaque(wm * FM * 2048 + short_chunk_at(r, h)), w_from = opaque(BM * 64 + wn * FN * 1024 + pair_at(r, h));
    auto read = [&](Fragments& f, const uint8_t* from) SLLM_INLINE {
#pragma unroll
        for (int n = 0; n < FN; ++n) f.w[n] = lds_read<u32x4>(from, w_from + n * 1024);
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int i = 0; i < 2; ++i) f.x[m][i] = lds_read<u32x4>(from, (x_from ^ i * 32) + m * 2048);
    };
    auto multiply = [&](const Fragments& f, const Scales& s, auto which) SLLM_INLINE {
        constexpr int i = decltype(which)::value;
        pin(acc);
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) {
                const i32x8 x = {(int)f.x[m][0][0], (int)f.x[m][0][1], (int)f.x[m][0][2], (int)f.x[m][0][3],
                                 (int)f.x[m][1][0], (int)f.x[m][1][1], (int)f.x[m][1][2], (int)f.x[m][1][3]};
                acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fragment(f.w[n]), x, acc[n][m], 4, 0, i % 2 * 2, s.w[n][i / 2],
                                                                            i % 2 * 2, s.x[m][i / 2]);
            }
        pin(acc);
    };
    // While one stage is multiplied the next is read, past the barrier where its loads have
    // landed; from that barrier on the buffer of the first is free, and takes the loads of
    // the fourth stage ahead.
    Fragments f0, f1;
    Scales now;
    auto stage = [&](uint64_t at, uint8_t* here, const uint8_t* next_one, const Fragments& f, Fragments& next, auto which, auto more) SLLM_INLINE {
        wait_but_loads<2 * kLoads>();  // younger than the next stage's: those of the two after it
        barrier();
        read(next, next_one);
        load(at + 4 * kStageBlocks, here);
        more();
        multiply(f, now, which);
    };
    auto group = [&](uint32_t t, uint8_t* s_now, uint8_t* s_next) SLLM_INLINE {
        const uint64_t at = (uint64_t)t * kGroupBlocks;
        const auto none = []() SLLM_INLINE {};
        const std::integral_constant<int, 0> i0;
        const std::integral_constant<int, 1> i1;
        const std::integral_constant<int, 2> i2;
        const std::integral_constant<int, 3> i3;
        stage(at, b0, b1, f0, f1, i0, [&]() SLLM_INLINE { load_scales(t + 1, s_next); });
        stage(at + 2, b1, b2, f1, f0, i1, none);
        stage(at + 4, b2, b3, f0, f1, i2, none);
        stage(at + 6, b3, b0, f1, f0, i3, none);
        read_scales(now, at, s_now, 1);
        stage(at + 8, b0, b1, f0, f1, i0, none);
        stage(at + 10, b1, b2, f1, f0, i1, none);
        stage(at + 12, b2, b3, f0, f1, i2, none);
        stage(at + 14, b3, b0, f1, f0, i3, none);
        read_scales(now, at + kGroupBlocks, s_next, 0);
    };
    if (t0 < t1) {
        const uint64_t at = (uint64_t)t0 * kGroupBlocks;
        load_scales(t0, s0);
        load(at, b0);
        load(at + 2, b1);
        load(at + 4, b2);
        load(at + 6, b3);
        wait_but_loads<3 * kLoads>();
        barrier();
        read(f0, b0);
        read_scales(now, at, s0, 0);
        for (uint32_t t = t0; t < t1; t += 2) {
            group(t, s0, s1);
            if (t + 1 < t1) group(t + 1, s1, s0);
        }
        wait_but_loads<0>();
        barrier();
    }
    // the output goes through two stages' buffers
    constexpr uint32_t kTurns = kStageBytes / kTurnBytes;
    static_assert(kWaves <= 2 * kTurns, "");
    uint8_t* const turn = wave < kTurns ? b0 + wave * kTurnBytes : b1 + (wave - kTurns) * kTurnBytes;
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 32, j0 + wn * FN * 32, out, turn);
}

}  // namespace

int32_t launch_mx8(const NarrowArgs& a, uint32_t tile, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, {
        T* to = static_cast<T*>(out);
        if (tile == kLargeTile)
            mx8_product<kLargeTile, kLargeTile, 2, 4, T><<<grid, 512, 0, stream>>>(a, to);
        else
            mx8_product<kSmallTile, kSmallTile, 2, 2, T><<<grid, 256, 0, stream>>>(a, to);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
