// gfx950 kernel of dy times an MX FP4 weight: the gradient by a product's input.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

constexpr uint32_t kStep = kWideStep;

// out[m][k] = sum over j of dy[m][j] W[j][k], in 32 bits.  4096 x 8192 by 8192 takes 445
// to 490 us, 1.15 to 1.2 PF/s: the matrix cores are busy 53 % of the cycles at 1.95 to
// 2.05 GHz; LDS is in use 41 %, a third of that conflicts, whose cause, the stores of W
// or the transposing reads, has not been separated.  2048 x 11008 by 4096 takes 174 us, in
// halves (128 tiles on 256 CUs), and 13.5 to join them.
//
// The depth runs along W's columns here, while its blocks lie along the rows.  So W
// is expanded on its way to LDS, by lanes that keep its codes two stages ahead, and
// a read that transposes gives each lane a column.  Otherwise as the product by
// W's rows.  X: what dy is multiplied in.
template <int BM, int BN, int WM, int WN, typename X, typename T>
__global__ __launch_bounds__(WM* WN * 64, 2) void grad_product(WideArgs a, T* out) {
    constexpr int kThreads = WM * WN * 64, kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kLoads = BM / 8 / kWaves;               // loads of x a wave issues a stage
    constexpr int kWords = BN * kStep / 8 / kThreads;     // of W, eight codes each, that a lane expands a stage
    constexpr int kPitch = BN * 2 + 32;                   // bytes of a row of W's tile in LDS
    constexpr int kXBytes = BM * kStep * 2, kWBytes = kStep * kPitch;
    constexpr bool kHalf = __is_same(X, _Float16);
    // The stages are variables of their own: the compiler then sees that loads
    // into one do not touch what is read from another.
    __shared__ __align__(16) uint8_t x0[kXBytes], x1[kXBytes];
    __shared__ __align__(16) uint8_t w0[kWBytes], w1[kWBytes];
    __shared__ uint32_t ranges[kHalf ? BM : 1];
    __shared__ uint32_t marks[kHalf ? kMarkWords : 1];  // stages with blocks of W that are added afterwards
    uint8_t* const x_ring[2] = {x0, x1};
    uint8_t* const w_ring[2] = {w0, w1};
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t r = lane & 31, h = lane >> 5;
    const void* const zeros = zero_vector();
    const Tile tile = tile_of(blockIdx.x, a.tiles_m, a.tiles_j);
    const uint64_t m0 = (uint64_t)tile.m * BM, j0 = (uint64_t)tile.j * BN;
    // the parts of x take a piece of W in turn: it comes from memory once, then from L2
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
    const uint16_t* x_at[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) x_at[q] = a.x + min(m0 + (q * kWaves + wave) * 8 + lane / 8, a.m - 1) * a.x_stride + x_col;
    auto load_x = [&](uint32_t t, uint8_t* to) SLLM_INLINE {
        const uint64_t d = (uint64_t)(t / a.parts) * kStep, at = t % a.parts * a.part_stride + d;
        const bool inside = d + x_col < a.depth;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const void* p = x_at[q] + at;
            load_to_lds(inside ? p : zeros, to, (q * kWaves + wave) * 1024);
        }
    };
    // The part of a block a lane expands, of two stages.  Past the end
    // of the depth x is zero, so any codes do under a finite scale.
    static_assert(kWords == 2 || kWords == 4, "");
    typedef uint32_t words __attribute__((ext_vector_type(kWords)));
    words codes[2];
    uint32_t scales[2];
    constexpr uint32_t kParts = 4 / kWords, kRowLanes = BN / 32 * kParts;
    const uint32_t w_row = tid / kRowLanes, w_block = tid % kRowLanes / kParts, w_part = tid % kParts;
    const uint64_t w_at = min(j0 / 32 + w_block, a.w_blocks - 1);
    auto load_w = [&](uint32_t t, int to) SLLM_INLINE {
        const uint64_t row = min((uint64_t)(min(t, t1 - 1) / a.parts) * kStep + w_row, a.w_rows - 1);
        codes[to] = reinterpret_cast<const words*>(a.w_codes + row * a.w_blocks + w_at)[w_part];
        scales[to] = a.w_scales[row * a.w_scale_pitch + w_at];
    };
    // W's tile in LDS: rows of the depth by the tile's columns, whose order
    // changes from block to block so that a wave's stores reach all banks.
    uint32_t w_to[kWords];
#pragma unroll
    for (uint32_t w = 0; w < kWords; ++w)
        w_to[w] = opaque(w_row * kPitch + w_block * 64 + ((w_part * kWords + w) ^ (w_block & 3)) * 16);
    auto store_w = [&](uint32_t t, int from, uint8_t* to, auto type, bool beyond_only) SLLM_INLINE {
        typedef decltype(type) W;
        const bool inside = (uint64_t)(t / a.parts) * kStep + w_row < a.w_rows;
        const uint32_t s = inside ? scales[from] : 0;
        const float scale = __is_same(W, _Float16) ? half_scale(s) : mx_scale(s);
        bool left_out = false;
#pragma unroll
        for (uint32_t w = 0; w < kWords; ++w) {
            uint32_t c = codes[from][w];
            if constexpr (kHalf) {
                const bool beyond = inside & beyond_half(s, c);
                if (__is_same(W, _Float16) ? beyond : beyond_only && !beyond) c = 0;
                left_out |= beyond;
            }
            lds_write(to, w_to[w], expand8<W>(c, scale));
        }
        if (__is_same(W, _Float16) && __any(left_out)) mark_stage(marks, t);
    };

    // (Filled through a reference: a returned structure makes its reads' alias
    // information useless, and they wait for every load under way.)
    struct Fragments {
        u32x4 x[FM], w[FN];
    };
    // Step s of a stage is, in lane (r, h), eight of the depth from 32 h + 8 s.
    // Of W four rows of the tile and 16 columns are read by 16 lanes, transposed:
    // a lane gets a column.
    const uint32_t x_from = opaque(wm * FM * 4096 + chunk_at(r, 4 * h));
    uint32_t w_from[FN];
#pragma unroll
    for (int n = 0; n < FN; ++n) {
        const uint32_t b = wn * FN + n, l = lane & 15, piece = ((lane >> 4 & 1) * 2 + (l >> 1 & 1)) ^ (b & 3);
        w_from[n] = opaque((32 * h + (l >> 2)) * kPitch + b * 64 + piece * 16 + (l & 1) * 8);
    }
    auto read = [&](Fragments& f, const uint8_t* x_now, const uint8_t* w_now, uint32_t s) SLLM_INLINE {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            const lds_u8* const p = (const lds_u8*)w_now + w_from[n] + 8 * s * kPitch;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * kPitch));
            f.w[n] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
        for (int m = 0; m < FM; ++m) f.x[m] = lds_read<u32x4>(x_now, (x_from ^ s * 16) + m * 4096);
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
    Fragments f0, f1;
    auto stage = [&](uint32_t t, auto which) SLLM_INLINE {
        constexpr int i = decltype(which)::value;  // t's buffers
        uint8_t* const here = x_ring[i];
        read(f1, here, w_ring[i], 1);
        multiply(f0);
        read(f0, here, w_ring[i], 2);
        multiply(f1);
        read(f1, here, w_ring[i], 3);
        store_w(t + 1, i ^ 1, w_ring[i ^ 1], X(), false);
        multiply(f0);
        wait_but_loads<0>();
        barrier();
        load_w(t + 3, i ^ 1);
        if (t + 2 < t1) load_x(t + 2, here);
        read(f0, x_ring[i ^ 1], w_ring[i ^ 1], 0);
        multiply(f1);
    };
    if constexpr (kHalf) {
        if (tid < kMarkWords) marks[tid] = 0;
        __syncthreads();  // before the first piece of W may mark its stage
    }
    if (t0 < t1) {
        load_w(t0, 0);
        load_w(t0 + 1, 1);
        load_x(t0, x0);
        store_w(t0, 0, w0, X(), false);
        wait_but_loads<0>();
        barrier();
        load_w(t0 + 2, 0);
        if (t0 + 1 < t1) load_x(t0 + 1, x1);
        read(f0, x0, w0, 0);
        for (uint32_t t = t0; t < t1; t += 2) {
            stage(t, std::integral_constant<int, 0>());
            if (t + 1 < t1) stage(t + 1, std::integral_constant<int, 1>());
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
            load_x(t, x0);
            load_w(t, 0);
            store_w(t, 0, w0, __bf16(), !again);
            wait_but_loads<0>();
            barrier();
#pragma unroll
            for (uint32_t s = 0; s < 4; ++s) {
                read(f0, x0, w0, s);
#pragma unroll
                for (int m = 0; m < FM; ++m) {
                    u32x4 hi, lo;
                    split_half(f0.x[m], hi, lo);
#pragma unroll
                    for (int n = 0; n < FN; ++n)
                        acc[n][m] = product<__bf16>(f0.w[n], lo, product<__bf16>(f0.w[n], hi, acc[n][m]));
                    pin(acc);
                }
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
            grad_product<kLargeTile, kLargeTile, 2, 4, X, T><<<grid, 512, 0, stream>>>(a, to);
        else if (tile_m == kSmallTile)
            grad_product<kSmallTile, kSmallTile, 2, 2, X, T><<<grid, 256, 0, stream>>>(a, to);
        else if (tile_m == 64)
            grad_product<64, kSmallTile, 2, 2, X, T><<<grid, 256, 0, stream>>>(a, to);
        else
            grad_product<32, kSmallTile, 1, 4, X, T><<<grid, 256, 0, stream>>>(a, to);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace

int32_t launch_grad(const WideArgs& a, bool half, uint32_t tile_m, uint32_t splits, void* out, uint32_t out_dtype,
                    hipStream_t stream) {
    return (half ? launch<_Float16> : launch<__bf16>)(a, tile_m, splits, out, out_dtype, stream);
}

}  // namespace sllm
