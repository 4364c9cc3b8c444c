// gfx950 kernels of products with an MX FP4 weight and an x of 16 or 32 bits.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStep = kWideStep;

// out[m][j] = sum over k of x[m][k] W[j][k], in 32 bits.  4096 x 8192 by 8192, two
// rounds of tiles, takes 405 to 475 us by card and load, 1.2 to 1.35 PF/s: the matrix
// cores are busy 62 % of the cycles, at the 1.95 GHz that power leaves (alone they reach
// 1.8 PF/s, at 1.9).  1999 x 5120 by 13824, 432 tiles on 256 CUs, takes 241 us and keeps
// them busy 50 %: a sixth of the two rounds is empty.  LDS is in use 16 to 19 % of the
// cycles, one access cycle in 50 a conflict.
//
// Both operands go to LDS by loads that pass no registers, two stages of 64 of the
// depth ahead.  W stays in four bits up to a lane's registers and becomes bfloat16
// there, exactly: a quarter of the loads and of the LDS traffic, for one conversion
// to a matrix instruction.  A wave makes 128 x 64 of a tile of 256 x 256, so that
// four fragments of x and two of W serve eight instructions; tiles with fewer rows
// and columns are for smaller problems.  X: what x is multiplied in.
template <int BM, int BN, int WM, int WN, typename X, typename T>
__global__ __launch_bounds__(WM* WN * 64, 2) void wide_product(WideArgs a, T* out) {
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kXLoads = BM / 8 / kWaves, kWLoads = BN / 16 / kWaves;
    constexpr int kXBytes = BM * kStep * 2, kWBytes = BN * 64, kScaleBytes = BN * 4;
    constexpr bool kHalf = __is_same(X, _Float16);
    constexpr int kScaleRows = BN / kWaves;  // whose scales a wave loads
    static_assert(kScaleRows <= 64, "");
    // The stages are variables of their own: the compiler then sees that loads
    // into one do not touch what is read from another.  W and its scales are of
    // two stages each.
    __shared__ __align__(16) uint8_t x0[kXBytes], x1[kXBytes];
    __shared__ __align__(16) uint8_t w0[kWBytes + kScaleBytes], w1[kWBytes + kScaleBytes];
    __shared__ uint32_t ranges[kHalf ? BM : 1];
    __shared__ uint32_t marks[kHalf ? kMarkWords : 1];  // stages with blocks of W that are added afterwards
    uint8_t* const x_ring[2] = {x0, x1};
    uint8_t* const w_ring[2] = {w0, w1};
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
    const uint16_t* x_at[kXLoads];
#pragma unroll
    for (int q = 0; q < kXLoads; ++q) x_at[q] = a.x + min(m0 + (q * kWaves + wave) * 8 + lane / 8, a.m - 1) * a.x_stride + x_col;
    auto load_x = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint32_t part = t / a.steps;
        const uint64_t d = (uint64_t)(t - part * a.steps) * kStep, at = part * a.part_stride + d;
        const bool inside = d + x_col < a.depth;
#pragma unroll
        for (int q = 0; q < kXLoads; ++q) {
            const void* p = x_at[q] + at;
            load_to_lds(inside ? p : zeros, to, (q * kWaves + wave) * 1024);
        }
    };
    // W's codes likewise, one load 16 rows x 128 of the depth, and four scale
    // bytes a row.  Past the end of the depth x is zero, so any codes do.
    const uint32_t w_block = lane % 4 ^ lane / 16;
    const u32x4* w_at[kWLoads];
#pragma unroll
    for (int q = 0; q < kWLoads; ++q) w_at[q] = a.w_codes + min(j0 + (q * kWaves + wave) * 16 + lane / 4, a.w_rows - 1) * a.w_blocks;
    const uint8_t* const scales_at = a.w_scales + min(j0 + wave * kScaleRows + lane % kScaleRows, a.w_rows - 1) * a.w_scale_pitch;
    auto load_w = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint64_t b0 = (uint64_t)(t % a.steps) * 2, b = min(b0 + w_block, a.w_blocks - 1);
#pragma unroll
        for (int q = 0; q < kWLoads; ++q) load_to_lds(w_at[q] + b, to, (q * kWaves + wave) * 1024);
        if (lane < kScaleRows) load_word_to_lds(scales_at + b0, to, kWBytes + wave * kScaleRows * 4);
    };

    // Of a stage, lane (r, h) has 32 of the depth of its rows: the block of W
    // that it expands as it goes, eight codes a step.
    // (Filled through a reference: a returned structure makes its reads' alias
    // information useless, and they wait for every load under way.)
    struct Weight {
        u32x4 codes[FN];
        float scale[FN];
    };
    const uint32_t w_from = opaque(wn * FN * 2048 + short_chunk_at(r, h)), scale_from = opaque(kWBytes + wn * FN * 128 + r * 4 + h);
    auto read_w = [&](Weight& w, uint32_t t, const uint8_t* from, uint32_t odd, auto type, bool beyond_only) SLLM_INLINE {
        const bool inside = (uint64_t)(t % a.steps) * 2 + h < a.w_blocks;  // scale bytes past the row's end may hold anything
        bool left_out = false;
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            w.codes[n] = lds_read<u32x4>(from, (w_from ^ odd * 32) + n * 2048);
            const uint8_t read = lds_read<uint8_t>(from, scale_from + n * 128 + odd * 2), s = inside ? read : 0;
            w.scale[n] = mx_scale(s);
            if constexpr (kHalf) {
                const u32x4 c = w.codes[n];
                const bool beyond = inside & beyond_half(s, c[0] | c[1] | c[2] | c[3]);
                if constexpr (__is_same(decltype(type), _Float16)) {
                    w.scale[n] = half_scale(s);
                    left_out |= beyond;
                    w.codes[n] = beyond ? u32x4{0, 0, 0, 0} : c;
                } else {
                    w.codes[n] = beyond_only && !beyond ? u32x4{0, 0, 0, 0} : c;
                }
            }
        }
        if (__is_same(decltype(type), _Float16) && __any(left_out)) mark_stage(marks, t);
    };

    struct Fragments {
        u32x4 x[FM], w[FN];
    };
    // Step s of a stage is, in lane (r, h), eight of the depth from 32 h + 8 s.
    const uint32_t x_from = opaque(wm * FM * 4096 + chunk_at(r, 4 * h));
    auto read = [&](Fragments& f, const uint8_t* from, const Weight& w, auto which) SLLM_INLINE {
        constexpr int s = decltype(which)::value;
#pragma unroll
        for (int m = 0; m < FM; ++m) f.x[m] = lds_read<u32x4>(from, (x_from ^ s * 16) + m * 4096);
#pragma unroll
        for (int n = 0; n < FN; ++n) f.w[n] = expand8<X>(w.codes[n][s], w.scale[n]);
    };
    bool fits = true;  // this lane's rows of x
    _Float16 factor[FM];
    float unit[FM];
    if constexpr (kHalf) {
        if (!a.ranges) find_tile_ranges<BM, kWaves * 64>(a, m0, t0, t1, ranges);
#pragma unroll
        for (int m = 0; m < FM; ++m) {
            const uint32_t row = (wm * FM + m) * 32 + r, range = a.ranges ? a.ranges[min(m0 + row, a.m - 1)] : ranges[row];
            fits &= row_fits(range);
            factor[m] = (_Float16)(float)(1 << row_shift(range));
            unit[m] = 1.0f / (1 << (row_shift(range) + kHalfShift));
        }
    }
    auto multiply = [&](const Fragments& f) SLLM_INLINE {
        u32x4 x[FM];
#pragma unroll
        for (int m = 0; m < FM; ++m) x[m] = kHalf ? __builtin_bit_cast(u32x4, __builtin_bit_cast(f16x8, f.x[m]) * factor[m]) : f.x[m];
        pin(acc);
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) acc[n][m] = product<X>(f.w[n], x[m], acc[n][m]);
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
    auto stage = [&](uint32_t t, auto which) SLLM_INLINE {
        constexpr int i = decltype(which)::value;  // t's place among the four stages that W's two buffers hold
        uint8_t* const here = x_ring[i % 2];
        read(f1, here, now, S1());
        multiply(f0);
        read(f0, here, now, S2());
        multiply(f1);
        read(f1, here, now, S3());
        multiply(f0);
        wait_but_loads<0>();
        barrier();
        read_w(now, t + 1, w_ring[(i + 1) / 2 % 2], (i + 1) % 2, X(), false);
        if (t + 2 < t1) load_x(t + 2, here);
        if (i % 2 && t + 3 < t1) load_w(t + 3, w_ring[i / 2]);
        read(f0, x_ring[(i + 1) % 2], now, S0());
        multiply(f1);
    };
    if (kHalf && tid < kMarkWords) marks[tid] = 0;  // a barrier before the first piece of W is read
    if (t0 < t1) {
        load_w(t0, w0);
        load_x(t0, x0);
        wait_but_loads<0>();
        barrier();
        load_x(t0 + 1, x1);
        if (t0 + 2 < t1) load_w(t0 + 2, w1);
        read_w(now, t0, w0, 0, X(), false);
        read(f0, x0, now, S0());
        for (uint32_t t = t0; t < t1; t += 4) {
            stage(t, S0());
            stage(t + 1, S1());
            if (t + 2 < t1) {
                stage(t + 2, S2());
                stage(t + 3, S3());
            }
        }
    }

    __syncthreads();  // the last stage's reads are done
    if constexpr (kHalf) {
        const bool again = __syncthreads_or(!fits);
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int m = 0; m < FM; ++m) acc[n][m] = again ? f32x16{} : acc[n][m] * unit[m];
        // All of W again, or what was left out of it.  With nothing to overlap, a stage
        // takes four times what it takes above.
        for (uint32_t t = t0; t < t1; ++t) {
            if (!again && !marked(marks, t)) continue;
            load_w(t & ~1u, w0);
            load_x(t, x0);
            wait_but_loads<0>();
            barrier();
            read_w(now, t, w0, t % 2, __bf16(), !again);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int m = 0; m < FM; ++m) {
                    u32x4 hi, lo;
                    split_half(lds_read<u32x4>(x0, (x_from ^ s * 16) + m * 4096), hi, lo);
#pragma unroll
                    for (int n = 0; n < FN; ++n) {
                        const u32x4 w = expand8(now.codes[n][s], now.scale[n]);
                        acc[n][m] = product<__bf16>(w, lo, product<__bf16>(w, hi, acc[n][m]));
                    }
                    pin(acc);
                }
            __syncthreads();
        }
    }
    // the output goes through the stages' buffers, a part of one for each wave
    constexpr int kTurns = kXBytes / kTurnBytes;
    static_assert(kXBytes % kTurnBytes == 0 && kWBytes >= kTurnBytes && 2 * kTurns + 2 >= kWaves, "");
    const int turn_at = (int)wave % kTurns * kTurnBytes, turn_of = (int)wave / kTurns;
    uint8_t* const turn = (turn_of == 0 ? x0 : turn_of == 1 ? x1 : wave == 2 * kTurns ? w0 : w1) + (turn_of < 2 ? turn_at : 0);
    store_tile<FM, FN>(acc, a.out_args, m0 + wm * FM * 32, j0 + wn * FN * 32, out, turn);
}

template <typename X>
int32_t launch(const WideArgs& a, uint32_t tile_m, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream) {
    const dim3 grid(a.tiles_m * a.tiles_j, splits);
    SLLM_BY_DTYPE(out_dtype, T, {
        T* to = static_cast<T*>(out);
        if (tile_m == kLargeTile)
            wide_product<kLargeTile, kLargeTile, 2, 4, X, T><<<grid, 512, 0, stream>>>(a, to);
        else if (tile_m == kSmallTile)
            wide_product<kSmallTile, kSmallTile, 2, 2, X, T><<<grid, 256, 0, stream>>>(a, to);
        else if (tile_m == 64)
            wide_product<64, kSmallTile, 2, 2, X, T><<<grid, 256, 0, stream>>>(a, to);
        else
            wide_product<32, kSmallTile, 1, 4, X, T><<<grid, 256, 0, stream>>>(a, to);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace

int32_t launch_wide(const WideArgs& a, bool half, uint32_t tile_m, uint32_t splits, void* out, uint32_t out_dtype,
                    hipStream_t stream) {
    return (half ? launch<_Float16> : launch<__bf16>)(a, tile_m, splits, out, out_dtype, stream);
}

}  // namespace sllm
