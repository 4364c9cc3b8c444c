// gfx950 kernels of products with few rows of x and an MX FP4 weight: decoding.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "products.hpp"

namespace sllm {

namespace {

// The upper halves of two floats, a's first: their leading bfloat16s.
__device__ __forceinline__ uint32_t upper_halves(float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
}

// Eight elements of x as the bfloat16 vectors whose sum they are, as far down as
// bfloat16's smallest step: each but the last takes the leading eight bits of what
// is left.  An infinity or a NaN is whole in the first.
template <typename X>
struct Parts {
    static constexpr int n = sizeof(X) == 4 ? 3 : 2;
    bf16x8 v[n];

    __device__ __forceinline__ void set(const X (&x)[8]) {
        u32x4 o[n];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            // quiet a NaN: its payload may be all in the lower half
            float a = __builtin_canonicalizef(to_f32(x[e])), b = __builtin_canonicalizef(to_f32(x[e + 1]));
            constexpr int kNotFinite = 0x207;  // NaN, -inf and +inf as v_cmp_class has them
            const bool a_ends = __builtin_amdgcn_classf(a, kNotFinite), b_ends = __builtin_amdgcn_classf(b, kNotFinite);
#pragma unroll
            for (int i = 0; i < n; ++i) {
                o[i][e / 2] = upper_halves(a, b);
                if (i + 1 == n) break;
                a -= __uint_as_float(__float_as_uint(a) & 0xffff0000);
                b -= __uint_as_float(__float_as_uint(b) & 0xffff0000);
                if (i == 0) {
                    a = a_ends ? 0.0f : a;
                    b = b_ends ? 0.0f : b;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = __builtin_bit_cast(bf16x8, o[i]);
    }
};

template <>
struct Parts<__bf16> {
    static constexpr int n = 1;
    bf16x8 v[1];

    __device__ __forceinline__ void set(const __bf16 (&x)[8]) { __builtin_memcpy(v, x, sizeof v); }
};

// X, or four bits of it a byte
template <typename X>
struct Element {
    typedef X type;
};
template <>
struct Element<void> {
    typedef uint8_t type;
};

// Eight elements of a row from column c, those past the end zero.
template <typename X>
struct Eight {
    X e[8];

    __device__ __forceinline__ void load(const X* row, uint64_t c, uint64_t cols, bool vector) {
        if (vector && c + 8 <= cols) {
            u32x4 raw[sizeof(X) / 2];
#pragma unroll
            for (uint32_t i = 0; i < sizeof(X) / 2; ++i) raw[i] = reinterpret_cast<const u32x4*>(row + c)[i];
            __builtin_memcpy(e, raw, sizeof e);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? row[c + i] : (X)0.0f;
        }
    }
};

// out[m][j] = sum over k of x[m][k] W[j][k] for few rows of x, in 32 bits.  Bound by
// reading W from memory, and for small ones by the launch and the way there: one
// row by 32000 x 4096 (70 MB) 17.5 us, 4.0 TB/s, by 11008 x 4096 9.6, by 4096 x 4096
// 5.4.  With 16 rows x is read as often as W has columns, and bounds it.
//
// A workgroup makes 16 columns of the output, its waves each a run of the depth;
// their sums are joined in LDS, first to last.  Of a step of 128 of the depth,
// lane (r, g) loads block g of row r: the order in which the matrix instructions
// take a step's columns does not matter as long as both sides have the same.
//
// Four steps, a group, are loaded together, and up to two groups are under way.  A
// row's 16 scale bytes of a group are one load, four bytes a lane, which the
// lanes then pass around: a load a step kept the address units as long as that
// step's codes did.  x comes a step ahead, and only in the lanes that have a row
// of it.
constexpr uint32_t kGroupBlocks = 16;

// A row's codes and scales of a group.
struct Group {
    u32x4 codes[4];
    uint32_t scales;

    __device__ __forceinline__ void load(const u32x4* row, const uint8_t* scale_row, uint32_t group, uint32_t g, uint64_t blocks) {
        const uint64_t b = (uint64_t)group * kGroupBlocks;
#pragma unroll
        for (int u = 0; u < 4; ++u) codes[u] = row[min(b + 4 * u + g, blocks - 1)];
        scales = *reinterpret_cast<const uint32_t*>(scale_row + b + 4 * g);
    }
};

// The scale bytes of step u, of what the four lanes of a row loaded: lane (r, u) has them.
__device__ __forceinline__ uint32_t step_scales(uint32_t scales, int u, uint32_t r) {
    return (uint32_t)__builtin_amdgcn_ds_bpermute((u * 16 + r) * 4, scales);
}

// Word j of lane (r, g) becomes word g of lane (r, j): a 4 x 4 transpose among the
// four lanes of a row, by swaps of half waves and of neighbouring rows of 16
// lanes.  Then eight columns from 32 j + 8 g are lane (r, g)'s, and one load of x
// takes 64 bytes of each row, not 16 bytes out of every 64.
__device__ __forceinline__ u32x4 transpose4(u32x4 v) {
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false));
    const u32x2 c = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false));
    const u32x2 d = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false));
    return u32x4{c[0], c[1], d[0], d[1]};
}

// Rows of x a tile of 16 columns of the second operand holds.  A matrix
// instruction takes 16 whatever they are, so where x has one row, or up to four,
// a load fetches 16, or four, pieces of the depth for each, side by side, and all
// but one piece are masked for each instruction: a 16th, or a quarter, of the
// loads of x and of its splitting into parts.  The pieces' sums are columns of
// their own until the end.  One row by 32000 x 4096: 17.5 us, in quarters 19.3, by 16
// rows 26.2; four rows by 11008 x 4096: 10.0 and 12.9.
template <typename X, int Rows, int MT>
__global__ __launch_bounds__(1024) void skinny_product(SkinnyArgs a) {
    extern __shared__ float sums[];
    constexpr bool kMx = __is_same(X, void);
    constexpr uint32_t kPieces = 16 / Rows;
    static_assert((Rows == 1 || Rows == 4 || Rows == 16) && (Rows == 16 || MT == 1), "");
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t waves = blockDim.x >> 6, r = lane & 15, g = lane >> 4;
    const uint64_t j0 = (uint64_t)block_index() * 16;
    const uint32_t g0 = (uint64_t)a.groups * wave / waves, g1 = (uint64_t)a.groups * (wave + 1) / waves;

    f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4{0, 0, 0, 0};

    const uint64_t row = min(j0 + r, a.n - 1);
    const u32x4* const w_codes = a.w_codes + row * a.blocks;
    const uint8_t* const w_scales = a.w_scales + row * a.scale_pitch;
    bool has_x[MT];
    uint64_t x_row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        x_row[m] = m * 16 + r / kPieces;
        has_x[m] = x_row[m] < a.m;
        x_row[m] = min(x_row[m], a.m - 1);
    }
    constexpr int kRing = sizeof(typename Element<X>::type) == 4 ? 1 : 2;  // registers hold no more
    Group w[kRing];
    auto load_w = [&](uint32_t group, int to) SLLM_INLINE {
        if (group < g1) w[to].load(w_codes, w_scales, group, g, a.blocks);
    };
    auto run = [&](const auto& multiply) SLLM_INLINE {
#pragma unroll
        for (int i = 0; i < kRing; ++i) load_w(g0 + i, i);
        for (uint32_t group = g0; group < g1; group += kRing)
#pragma unroll
            for (int i = 0; i < kRing; ++i) {
                if (group + i >= g1) break;
                multiply(group + i, w[i], i);
                load_w(group + i + kRing, i);
            }
    };
    if constexpr (kMx) {
        u32x4 x[2][MT] = {};
        uint32_t scales[MT] = {};
        auto load_x = [&](uint32_t step, int to) SLLM_INLINE {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                if (has_x[m]) x[to][m] = static_cast<const u32x4*>(a.x)[x_row[m] * a.blocks + min((uint64_t)step * 4 + g, a.blocks - 1)];
        };
        if (g0 < g1) load_x(g0 * 4, 0);
        run([&](uint32_t group, const Group& held, int) SLLM_INLINE {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                scales[m] = *reinterpret_cast<const uint32_t*>(a.x_scales + x_row[m] * a.scale_pitch + group * kGroupBlocks + 4 * g);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                load_x(group * 4 + u + 1, (u + 1) % 2);
                // past the end of the depth x is zero, and the scales must be numbers
                const uint32_t mask = (uint64_t)group * kGroupBlocks + 4 * u + g < a.blocks ? ~0u : 0;
                const uint32_t ws = step_scales(held.scales, u, r) >> (8 * g) & mask;
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    acc[m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(held.codes[u]), fragment(x[u % 2][m] & mask), acc[m],
                                                                              4, 4, 0, ws, 0, step_scales(scales[m], u, r) >> (8 * g) & mask);
            }
        });
    } else {
        const X* x[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) x[m] = static_cast<const X*>(a.x) + x_row[m] * a.x_stride;
        // the products of step u, j of a group with the parts of x
        auto multiply = [&](uint32_t group, int u, int j, uint32_t codes, uint32_t scales, const Parts<X> (&p)[MT]) SLLM_INLINE {
            const bool inside = (uint64_t)group * kGroupBlocks + 4 * u + j < a.blocks;  // else x is zero, any number does
            const bf16x8 wide = __builtin_bit_cast(bf16x8, expand8(codes, mx_scale(inside ? scales >> (8 * j) & 0xff : 0)));
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < Parts<X>::n; ++i) {
                    u32x4 v = __builtin_bit_cast(u32x4, p[m].v[i]);
                    if (Rows == 1) v = r == uint32_t(u * 4 + j) ? v : u32x4{0, 0, 0, 0};
                    if (Rows == 4) v = r % 4 == uint32_t(j) ? v : u32x4{0, 0, 0, 0};
                    acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide, __builtin_bit_cast(bf16x8, v), acc[m], 0, 0, 0);
                }
        };
        if constexpr (Rows < 16) {
            // x of a group at a time, as far ahead as the weight
            constexpr int kLoads = Rows;
            Eight<X> raw[kRing][kLoads] = {};
            auto load_x = [&](uint32_t group, int to) SLLM_INLINE {
                if (group >= g1 || !has_x[0]) return;
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
                    raw[to][q].load(x[0], (uint64_t)group * 512 + q * 128 + r % kPieces * 32 + 8 * g, a.depth, a.vector);
            };
#pragma unroll
            for (int i = 0; i < kRing; ++i) load_x(g0 + i, i);
            run([&](uint32_t group, const Group& held, int at) SLLM_INLINE {
                Parts<X> p[kLoads][1];
#pragma unroll
                for (int q = 0; q < kLoads; ++q) p[q][0].set(raw[at][q].e);
                load_x(group + kRing, at);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const u32x4 codes = transpose4(held.codes[u]);
                    const uint32_t scales = step_scales(held.scales, u, r);
#pragma unroll
                    for (int j = 0; j < 4; ++j) multiply(group, u, j, codes[j], scales, p[u % kLoads]);
                }
            });
        } else {
            Eight<X> raw[2][4][MT] = {};
            auto load_x = [&](uint32_t step, int to) SLLM_INLINE {
                const uint64_t c = (uint64_t)step * 128 + 8 * g;
                const bool whole = a.vector && (uint64_t)(step + 1) * 128 <= a.depth;
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if (has_x[m])
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (whole)
                                raw[to][j][m].load(x[m], c + j * 32, ~0ull, true);
                            else
                                raw[to][j][m].load(x[m], c + j * 32, a.depth, a.vector);
                        }
            };
            if (g0 < g1) load_x(g0 * 4, 0);
            run([&](uint32_t group, const Group& held, int) SLLM_INLINE {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (u < 3 || group + 1 < g1) load_x(group * 4 + u + 1, (u + 1) % 2);
                    const u32x4 codes = transpose4(held.codes[u]);
                    const uint32_t scales = step_scales(held.scales, u, r);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        Parts<X> p[MT];
#pragma unroll
                        for (int m = 0; m < MT; ++m) p[m].set(raw[u % 2][j][m].e);
                        multiply(group, u, j, codes[j], scales, p);
                    }
                }
            });
        }
    }
    if constexpr (Rows < 16) {
#pragma unroll
        for (uint32_t d = 1; d < kPieces; d *= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[0][i] += __shfl_xor(acc[0][i], d);
    }

    // lane (r, g) has columns 4 g .. + 3 of the tile for row r / kPieces of x
    constexpr uint32_t kCols = 16, kSums = Rows * MT * kCols;
#pragma unroll
    for (int m = 0; m < MT; ++m)
        if (r % kPieces == 0) *reinterpret_cast<f32x4*>(sums + wave * kSums + (m * 16 + r / kPieces) * kCols + g * 4) = acc[m];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kSums; i += blockDim.x) {
        const uint64_t m = i / kCols, j = j0 + i % kCols;
        if (m >= a.m || j >= a.n) continue;
        float sum = 0;
        for (uint32_t w = 0; w < waves; ++w) sum += sums[w * kSums + i];
        const uint64_t at = m * a.out_stride + j;
        if (a.out_dtype == SLLM_DTYPE_F32)
            static_cast<float*>(a.out)[at] = sum;
        else if (a.out_dtype == SLLM_DTYPE_F16)
            static_cast<_Float16*>(a.out)[at] = from_f32<_Float16>(sum);
        else
            static_cast<__bf16*>(a.out)[at] = from_f32<__bf16>(sum);
    }
}

template <typename X, int Rows, int MT>
void launch(const SkinnyArgs& a, hipStream_t stream) {
    const uint32_t grid = (uint32_t)((a.n + 15) / 16);
    // Enough waves to fill the GPU, two groups of the depth for each where there are
    // as many: one row by 32000 x 4096 17.5 us with four waves, 20.0 with eight; by
    // 1024 x 8192 5.9 with 16, 7.3 with four.
    uint32_t waves = 4;
    while (waves < 16 && (a.groups > waves * 2 || (grid * waves < 2048 && a.groups > waves))) waves *= 2;
    while (waves > 1 && a.groups < waves) waves /= 2;
    skinny_product<X, Rows, MT><<<grid_of(grid), waves * 64, waves * Rows * MT * 16 * 4, stream>>>(a);
}

}  // namespace

int32_t launch_skinny(const SkinnyArgs& a, hipStream_t stream) {
    if (a.x_scales && a.m <= 16)
        launch<void, 16, 1>(a, stream);
    else if (a.x_scales)
        launch<void, 16, 2>(a, stream);
    else
        SLLM_BY_DTYPE(a.x_dtype, X, {
            if (a.m == 1)
                launch<X, 1, 1>(a, stream);
            else if (a.m <= 4)
                launch<X, 4, 1>(a, stream);
            else
                launch<X, 16, 1>(a, stream);
        });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
