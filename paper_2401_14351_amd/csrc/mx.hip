// gfx950 kernels of MX FP4 matrices: quantisation, and the way a product is
// carried out (the products' own kernels are in gemm_*.hip).
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "operators.hpp"
#include "products.hpp"

namespace sllm {

namespace {

// ---------------------------------------------------------------------------
// Quantisation
// ---------------------------------------------------------------------------

// The scale byte of a block whose largest magnitude is `top` (0 to 254, or 255
// where it is no finite number): floor(log2 top) is the float's exponent
// field less 127, two less make 4 .. 8 of the largest element, and magnitudes
// below 2^-125 share the smallest scale.
__device__ __forceinline__ uint32_t block_scale(float top) {
    const uint32_t e = __float_as_uint(top) >> 23;
    return e == 255 ? 255 : e < 2 ? 0 : e - 2;
}

// x of the lane a DPP control names, among the four lanes of a block
template <int Ctrl>
__device__ __forceinline__ float quad(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), Ctrl, 0xF, 0xF, true));
}

// x is read once and its 4.25 bits a value written once; bound by memory (11008
// x 4096 in bfloat16, 90 MB in and 24 MB out, in 23.6 us, 4.8 TB/s; in 18.4 where
// the last-level cache still has x; two loads a lane under way take 25.8).  Four
// lanes a block, eight columns each: a lane's loads are 16 bytes wide, neighbours' codes
// are neighbouring words, and a block's largest magnitude is two lane exchanges
// away.  Elements are rounded to nearest even by the conversion instruction.
// `lanes` of them take a row at a time.  Vec: rows start on 16 bytes and end on a
// multiple of eight columns; else elements are loaded one by one.
template <bool Vec, typename T>
__global__ __launch_bounds__(256) void mx_quantize(const T* src, uint64_t stride, uint64_t rows, uint32_t cols, uint32_t lanes,
                                                   uint8_t* codes, uint8_t* scales) {
    const uint64_t row = (uint64_t)block_index() * (256 / lanes) + threadIdx.x / lanes;
    if (row >= rows) return;
    const uint32_t blocks = (cols + 31) / 32, pitch = (blocks + 15) / 16 * 16;
    const T* x = src + row * stride;
    uint32_t* out = reinterpret_cast<uint32_t*>(codes + row * blocks * 16);
    uint8_t* scale_row = scales + row * pitch;
    for (uint32_t i = threadIdx.x % lanes; i < pitch * 4; i += lanes) {
        const uint32_t b = i / 4, c = i * 8;
        if (b >= blocks) {
            if (i % 4 == 0) scale_row[b] = 0;
            continue;
        }
        T e[8];
        if (Vec && c < cols) {
            u32x4 raw[sizeof(T) / 2];
#pragma unroll
            for (uint32_t j = 0; j < sizeof(T) / 2; ++j) raw[j] = reinterpret_cast<const u32x4*>(x + c)[j];
            __builtin_memcpy(e, raw, sizeof e);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) e[j] = c + j < cols ? x[c + j] : (T)0.0f;
        }
        // magnitudes as integers order as the numbers do, infinities and NaN above all others
        uint32_t top = 0;
        float v[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            v[j] = to_f32(e[j]);
            top = max(top, __float_as_uint(v[j]) & 0x7fffffff);
        }
        top = max(top, __float_as_uint(quad<0xB1>(__uint_as_float(top))));  // lanes 1 0 3 2
        top = max(top, __float_as_uint(quad<0x4E>(__uint_as_float(top))));  // lanes 2 3 0 1
        const uint32_t s = block_scale(__uint_as_float(top));
        const float f = mx_scale(s);
        uint32_t packed = 0;
        if (s != 255) {
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, v[0], v[1], f, 0);
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, v[2], v[3], f, 1);
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, v[4], v[5], f, 2);
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(packed, v[6], v[7], f, 3);
        }
        out[i] = packed;
        if (i % 4 == 0) scale_row[b] = s;
    }
}

}  // namespace

int32_t launch_quantize(const sllm_matrix& src, const sllm_mx& dst, hipStream_t stream) {
    const uint64_t vectors = mx_scale_pitch(src.cols) * 4;
    // Long rows take a workgroup (11008 rows of 4096 in 32 bits 39 us, a wave each
    // 44; 512 rows 3.7 and 6.1), short ones a wave (32000 of 768 in bfloat16 12, a
    // workgroup 18).
    const uint32_t lanes = vectors >= 256 ? 256 : 64;
    const dim3 grid = grid_of(ceil_div(src.rows, 256 / lanes));
    const uint64_t row_bytes = src.stride * (src.dtype == SLLM_DTYPE_F32 ? 4 : 2);
    const bool vec = src.cols % 8 == 0 && reinterpret_cast<uintptr_t>(src.data) % 16 == 0 && (src.rows == 1 || row_bytes % 16 == 0);
    uint8_t *codes = static_cast<uint8_t*>(dst.codes), *scales = static_cast<uint8_t*>(dst.scales);
    SLLM_BY_DTYPE(src.dtype, T, {
        const T* x = static_cast<const T*>(src.data);
        if (vec)
            mx_quantize<true, T><<<grid, 256, 0, stream>>>(x, src.stride, src.rows, (uint32_t)src.cols, lanes, codes, scales);
        else
            mx_quantize<false, T><<<grid, 256, 0, stream>>>(x, src.stride, src.rows, (uint32_t)src.cols, lanes, codes, scales);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

namespace {

// How a product is carried out, from its operands alone.
struct Plan {
    bool skinny = false;       // one launch, nothing staged
    uint32_t parts = 1;        // bfloat16 matrices that x is the sum of
    bool staged = false;       // x is written out as those first
    uint64_t depth = 0, cols = 0;
    uint64_t part_stride = 0;  // elements, of a staged x
    uint32_t tile_m = 0, tile_n = 0, steps = 0, splits = 1;
    uint32_t tiles_m = 0, tiles_j = 0;
    uint64_t x_bytes = 0, split_stride = 0, bytes = 0;
    bool ranges = false;       // those of a float16 x's rows are found first, to be
    uint64_t ranges_at = 0;    // here in the workspace
};

// Whether a product goes to the kernel of few rows.  It reads all of x for every
// 16 columns of the output, in registers and without a launch more, so it gains
// where rows and columns are few; measured in us here and by tiles, W 11008 x 4096
// unless said: bfloat16 5 rows 12.5 and 15.7, 8 rows 14.1 and 15.9, 16 rows 17.8 and
// 16.4, 16 rows by 32000 x 4096 42 and 30; float16 5 rows 17.2 and 18.1, 16 rows 20.1
// and 19.0, 16 rows by 16384 x 4096 25.2 and 21.5; float 16 rows 31 and 34, 16 rows by
// 32000 x 4096 71 and 67; MX FP4 16 rows 11.3 and 15.2, 32 rows 17.1 and 15.6;
// MX FP8 16 rows 12.4 and 17.9, by 16384 x 8192 31.7 and 33.8, more rows by 1024 x 4096
// 11 to 12 and 17.6, 32 by 4096 x 4096 13.8 and 17.6, by 4096 x 8192 26.5 and 21.3.
bool few_rows(const LinearLaunch& a) {
    if (a.grad) return false;
    if (a.x.fp8) return a.m <= 16 ? a.m * a.n <= 1 << 18 : a.m <= 32 && a.m * a.n * a.k <= 1 << 29;
    if (a.x.codes) return a.m <= 32 && a.m * a.n <= 1 << 18;
    if (a.m <= 4) return true;
    if (a.x.dtype == SLLM_DTYPE_F16) return a.m <= 16 && a.n <= 8192;
    return a.m <= 16 && a.m * a.n <= (a.x.dtype == SLLM_DTYPE_F32 ? 1 << 18 : 1 << 17);
}

Plan plan_linear(const LinearLaunch& a) {
    Plan p;
    p.depth = a.grad ? a.n : a.k;
    p.cols = a.grad ? a.k : a.n;
    p.skinny = few_rows(a);
    if (!p.depth || !a.m || !p.cols || p.skinny) return p;
    if (!a.x.codes) p.parts = a.x.dtype == SLLM_DTYPE_F32 ? 3 : 1;
    // The kernel reads x in aligned vectors of eight.
    p.staged = !a.x.codes && (p.parts > 1 || p.depth % 8 || (a.m > 1 && a.x.stride % 8) ||
                              reinterpret_cast<uintptr_t>(a.x.data) % 16);
    p.part_stride = (p.depth + 7) / 8 * 8;
    const uint32_t step = a.x.codes ? kNarrowStep : kWideStep;
    p.steps = (uint32_t)ceil_div(p.depth, step);
    if (!a.x.codes) p.steps += p.steps % 2;
    const auto tiles = [&](uint32_t rows, uint32_t cols) { return ceil_div(a.m, rows) * ceil_div(p.cols, cols); };
    const uint64_t depth = (uint64_t)p.steps * p.parts * step, large = tiles(kLargeTile, kLargeTile);
    const bool tall = a.m > kSmallTile;
    // Large tiles read the least per product, and serve where most CUs get one (in
    // us, large and small: 432 tiles 251 and 279, 172 tiles 93 and 97, MX FP4 39 and
    // 45), or half of one that is deep enough to pay for the join (128 tiles of a
    // depth of 11008: 180 and 208, MX FP4 73 and 81; of 4096 by 86 tiles 65 and 61).
    // Small ones are 32 or 64 rows tall where there are no more, since the rows past
    // the last cost as much (16 rows by 11008 x 4096: 32 tall 16.4, 64 18.7, 128 21.9;
    // 64 rows: 25.2, 21.0, 24.9), and 32 for problems of few stages of 128 x 128 x 64,
    // which would leave CUs empty (400 stages, 700 x 700 x 700: 32 tall 12.1, 64 14.2,
    // 128 18.3; 4096, 1000 x 2000 x 2000: 20.3, 26.0, 25.9; 6144, 300 x 4096 x 4096:
    // 34.2, 27.5, 29.2; 8192, 512 x 4096 x 4096: 38.5, 34.4, 33.5).  They split the
    // depth until there are two for each CU, of 512 of it at least: half as many take
    // 64 rows by 4096 x 4096 from 17.6 to 19.1, 1024 of it 333 rows by 2047 x 1000 from
    // 15.3 to 20.1, 256 of it 64 rows by 4096 x 4096 to 22.9.  With both sides in MX
    // FP4 a tile is done four times as fast, and splits pay later.
    if (tall && large >= 160) {
        p.tile_m = p.tile_n = kLargeTile;
    } else if (tall && large >= 112 && depth >= 8192) {
        p.tile_m = p.tile_n = kLargeTile;
        p.splits = 2;
    } else {
        p.tile_n = kSmallTile;
        const bool short_tiles = a.m <= 32 || tiles(kSmallTile, kSmallTile) * p.steps * p.parts <= 4096;
        p.tile_m = a.x.codes ? kSmallTile : short_tiles ? 32 : a.m <= 64 ? 64 : kSmallTile;
        const uint64_t fill = a.x.codes ? 128 : 512, piece = a.x.codes ? 4096 : 512;
        p.splits = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>({fill / tiles(p.tile_m, p.tile_n), depth / piece, 16}));
    }
    p.tiles_m = (uint32_t)ceil_div(a.m, p.tile_m);
    p.tiles_j = (uint32_t)ceil_div(p.cols, p.tile_n);
    if (p.staged) p.x_bytes = (a.m * p.parts * p.part_stride * 2 + 255) / 256 * 256;
    p.split_stride = a.m * ((p.cols + 3) / 4 * 4);
    p.bytes = p.x_bytes + (p.splits > 1 ? p.splits * p.split_stride * 4 : 0);
    // A workgroup finds the ranges of its own piece of a float16 x where that is small;
    // with a kernel before (in us, 64 rows by 768 x 768, a piece of 48 KB, 10.3 and 11.4;
    // 1024 x 1024 x 1024, 64 KB, 16.7 and 17.7; 1000 x 2000 x 2000, 128 KB, 28.2 and 26.4;
    // 1024 x 4096 x 4096, 512 KB, 72 and 59).  Where x is copied first that goes along.
    constexpr uint64_t kOwnRanges = 64 << 10;
    p.ranges = !a.x.codes && a.x.dtype == SLLM_DTYPE_F16 &&
               (p.staged || ceil_div(p.steps, p.splits) * kWideStep * p.tile_m * 2 > kOwnRanges);
    p.ranges_at = p.bytes;
    if (p.ranges) p.bytes += a.m * 4;
    return p;
}

// x as the sum of `Parts` bfloat16 matrices: its leading eight bits, the eight
// after those, the rest, as far down as bfloat16's smallest step, 2^-133.  Of one part
// it is a copy of a bfloat16 x, for rows that do not start on 16 bytes.  The products
// then load x straight to LDS, and the parts are made once, not by every tile.  Bound by
// its launch or by memory: 333 x 2047 in 16 bits 3.7 us.
template <typename T, int Parts>
__global__ __launch_bounds__(256) void split_x(const T* x, uint64_t stride, uint64_t rows, uint64_t cols, uint64_t pitch,
                                               uint16_t* out) {
    const uint64_t vectors = pitch / 8, i = (uint64_t)block_index() * 256 + threadIdx.x;
    const uint64_t row = i / vectors, c = i % vectors * 8;
    if (row >= rows) return;
    uint16_t v[Parts][8];
    for (uint32_t e = 0; e < 8; ++e) {
        const T at = c + e < cols ? x[row * stride + c + e] : T(0);
        if constexpr (Parts == 1) {
            v[0][e] = at;
        } else {
            float f = at;
            for (int p = 0; p < Parts; ++p) v[p][e] = leading_bf16(f);
        }
    }
    for (int p = 0; p < Parts; ++p) {
        u32x4 o;
        for (int j = 0; j < 4; ++j) o[j] = v[p][2 * j] | (uint32_t)v[p][2 * j + 1] << 16;
        *reinterpret_cast<u32x4*>(out + (row * Parts + p) * pitch + c) = o;
    }
}

// The range of each row of a float16 x (products.hpp says of what), a wave each, or where
// rows are long a workgroup; with Copy each row is written to `out` too, as split_x does.
// Vec: rows start on 16 bytes.  Bound by memory: 4096 x 8192 15 us, 4.4 TB/s, 13 where the
// last-level cache has it; 64 x 4096 2.8; 333 x 2047 copied 4.2.
template <bool Vec, bool Copy, int Lanes>
__global__ __launch_bounds__(256) void find_ranges(const uint16_t* x, uint64_t stride, uint64_t rows, uint64_t cols, uint64_t pitch,
                                                   uint16_t* out, uint32_t* ranges) {
    __shared__ uint32_t waves[4];
    const uint64_t row = (uint64_t)block_index() * (256 / Lanes) + threadIdx.x / Lanes;
    const uint16_t* at = x + min(row, rows - 1) * stride;
    RowRange range;
    for (uint64_t c = threadIdx.x % Lanes * 8; c < cols; c += Lanes * 8) {
        u32x4 v;
        if (Vec && c + 8 <= cols) {
            v = *reinterpret_cast<const u32x4*>(at + c);
        } else {
            uint16_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? at[c + i] : 0;
            __builtin_memcpy(&v, e, sizeof v);
        }
        range.add(v);
        if (Copy && row < rows) *reinterpret_cast<u32x4*>(out + row * pitch + c) = v;
    }
    range.join(64);
    if constexpr (Lanes > 64) {
        if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = range.word();
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            range.top = max(range.top, waves[w] & 0xffff);
            range.bottom = min(range.bottom, waves[w] >> 16);
        }
    }
    if (threadIdx.x % Lanes == 0 && row < rows) ranges[row] = range.word();
}

// The sum of the splits' matrices, first to last, so that every call adds in the
// same order.  Bound by memory: two of 2048 x 4096 (67 MB in, 17 MB out) 13.5 us,
// 6.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void join_splits(const float* in, uint32_t splits, uint64_t split_stride, uint64_t rows,
                                                   uint64_t cols, T* out, uint64_t stride) {
    const uint64_t vectors = (cols + 3) / 4, i = (uint64_t)block_index() * 256 + threadIdx.x;
    const uint64_t row = i / vectors, c = i % vectors * 4;
    if (row >= rows) return;
    f32x4 sum = {0, 0, 0, 0};
    for (uint32_t s = 0; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(in + s * split_stride + i * 4);
    for (uint32_t e = 0; e < 4 && c + e < cols; ++e) out[row * stride + c + e] = from_f32<T>(sum[e]);
}

int32_t join(const Plan& p, const float* sums, uint32_t splits, const LinearLaunch& a, hipStream_t stream) {
    const dim3 blocks = grid_of(ceil_div(a.m * ceil_div(p.cols, 4), 256));
    SLLM_BY_DTYPE(a.out_dtype, T, (join_splits<T><<<blocks, 256, 0, stream>>>(sums, splits, p.split_stride, a.m, p.cols,
                                                                             static_cast<T*>(a.out), a.out_stride)));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

// x as the wide kernel reads it, written out in the workspace where it is not so already,
// and the ranges of a float16 one.
int32_t stage_x(const LinearLaunch& a, const Plan& p, void* workspace, WideArgs* w, hipStream_t stream) {
    w->x = static_cast<const uint16_t*>(a.x.data);
    w->x_stride = a.x.stride, w->part_stride = 0;
    w->ranges = nullptr;
    uint16_t* x = static_cast<uint16_t*>(workspace);
    if (p.staged) {
        w->x = x;
        w->x_stride = p.parts * p.part_stride;
        w->part_stride = p.part_stride;
    }
    const dim3 blocks = grid_of(ceil_div(a.m * p.part_stride / 8, 256));
    if (p.ranges) {
        uint32_t* ranges = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + p.ranges_at);
        const uint16_t* from = static_cast<const uint16_t*>(a.x.data);
        const bool vec = reinterpret_cast<uintptr_t>(from) % 16 == 0 && (a.m == 1 || a.x.stride % 8 == 0), wide = p.depth > 1024;
        const auto kernel = p.staged ? (vec ? (wide ? find_ranges<true, true, 256> : find_ranges<true, true, 64>)
                                            : (wide ? find_ranges<false, true, 256> : find_ranges<false, true, 64>))
                                     : (wide ? find_ranges<true, false, 256> : find_ranges<true, false, 64>);
        kernel<<<grid_of(ceil_div(a.m, wide ? 1 : 4)), 256, 0, stream>>>(from, a.x.stride, a.m, p.depth, p.part_stride, x, ranges);
        w->ranges = ranges;
    } else if (p.staged && p.parts == 1) {
        split_x<uint16_t, 1><<<blocks, 256, 0, stream>>>(static_cast<const uint16_t*>(a.x.data), a.x.stride, a.m, p.depth, p.part_stride, x);
    } else if (p.staged) {
        split_x<float, 3><<<blocks, 256, 0, stream>>>(static_cast<const float*>(a.x.data), a.x.stride, a.m, p.depth, p.part_stride, x);
    }
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

int32_t launch_tiled(const LinearLaunch& a, const Plan& p, void* workspace, hipStream_t stream) {
    OutArgs o{a.m, p.cols, a.out_stride, 0, 0};
    void* out = a.out;
    uint32_t dtype = a.out_dtype;
    if (p.splits > 1) {
        out = static_cast<uint8_t*>(workspace) + p.x_bytes;
        dtype = SLLM_DTYPE_F32;
        o.stride = (p.cols + 3) / 4 * 4;
        o.split_stride = p.split_stride;
    }
    o.vector = reinterpret_cast<uintptr_t>(out) % 16 == 0 && (a.m == 1 || o.stride * (dtype == SLLM_DTYPE_F32 ? 4 : 2) % 16 == 0);
    if (a.x.codes) {
        const NarrowArgs n{reinterpret_cast<const u32x4*>(a.x.codes), a.x.scales, reinterpret_cast<const u32x4*>(a.w_codes),
                           a.w_scales, a.m, a.n, mx_blocks(a.k), mx_scale_pitch(a.k), p.steps, p.tiles_m, p.tiles_j, o};
        SLLM_TRY((a.x.fp8 ? launch_mx8 : launch_narrow)(n, p.tile_n, p.splits, out, dtype, stream));
    } else {
        WideArgs w;
        SLLM_TRY(stage_x(a, p, workspace, &w, stream));
        w.m = a.m, w.depth = p.depth;
        w.parts = p.parts, w.steps = p.steps;
        w.w_codes = reinterpret_cast<const u32x4*>(a.w_codes);
        w.w_scales = a.w_scales;
        w.w_rows = a.n, w.w_blocks = mx_blocks(a.k), w.w_scale_pitch = mx_scale_pitch(a.k);
        w.tiles_m = p.tiles_m, w.tiles_j = p.tiles_j;
        w.out_args = o;
        SLLM_TRY((a.grad ? launch_grad : launch_wide)(w, a.x.dtype == SLLM_DTYPE_F16, p.tile_m, p.splits, out, dtype, stream));
    }
    return p.splits > 1 ? join(p, static_cast<const float*>(out), p.splits, a, stream) : SLLM_OK;
}

}  // namespace

// x in MX FP8 and a result in 32 bits.  The scaled matrix instruction adds products of eight
// elements of x at a time, and drops what is 2^-13 below the largest of them: 2^-17 of a
// sum's magnitudes at the most where they are normally distributed, far less than 16 bits
// tell, but more than 32 bits do.  x is then written out as bfloat16, which holds it, and
// multiplied so (4096 x 8192 by 28672 1.42 ms, in eight bits 0.83).
bool widened(const LinearLaunch& a) { return a.x.fp8 && a.out_dtype == SLLM_DTYPE_F32; }

LinearLaunch widen(const LinearLaunch& a, void* x) {
    LinearLaunch w = a;
    w.x = Operand{x, (a.k + 7) / 8 * 8, SLLM_DTYPE_BF16, nullptr, nullptr, false};
    return w;
}

uint64_t widened_bytes(const LinearLaunch& a) { return (a.m * ((a.k + 7) / 8 * 8) * 2 + 255) / 256 * 256; }

uint64_t linear_workspace(const LinearLaunch& a) {
    if (widened(a)) return widened_bytes(a) + plan_linear(widen(a, nullptr)).bytes;
    return plan_linear(a).bytes;
}

int32_t launch_linear(const LinearLaunch& a, void* workspace, hipStream_t stream) {
    if (widened(a) && a.k) {
        const LinearLaunch w = widen(a, workspace);
        const sllm_mx x{const_cast<uint8_t*>(a.x.codes), const_cast<uint8_t*>(a.x.scales), a.m, a.k};
        SLLM_TRY(launch_mx8_dequantize(x, sllm_matrix{workspace, a.m, a.k, w.x.stride, SLLM_DTYPE_BF16, 0}, stream));
        return launch_linear(w, static_cast<uint8_t*>(workspace) + widened_bytes(a), stream);
    }
    const Plan plan = plan_linear(a);
    if (plan.skinny && plan.depth) {
        const uint64_t row_bytes = a.x.stride * (a.x.dtype == SLLM_DTYPE_F32 ? 4 : 2);
        const bool vector = reinterpret_cast<uintptr_t>(a.x.data) % 16 == 0 && (a.m == 1 || row_bytes % 16 == 0);
        return launch_skinny(SkinnyArgs{a.x.codes ? a.x.codes : a.x.data, a.x.scales, a.x.fp8, a.m, a.n, a.k, a.x.stride, a.x.dtype, vector,
                                        reinterpret_cast<const u32x4*>(a.w_codes), a.w_scales, mx_blocks(a.k), mx_scale_pitch(a.k),
                                        (uint32_t)ceil_div(a.k, 512), a.out, a.out_stride, a.out_dtype}, stream);
    }
    if (plan.depth) return launch_tiled(a, plan, workspace, stream);
    // a depth of zero: sums of nothing
    return join(plan, nullptr, 0, a, stream);
}

}  // namespace sllm
