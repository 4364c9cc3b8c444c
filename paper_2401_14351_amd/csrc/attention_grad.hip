// gfx950 kernels of the gradients of attention over packed sequences.
#include <algorithm>

#include "attention.hpp"
#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"

namespace sllm {

namespace {

constexpr int kWaves = 4, kWaveRows = 32, kRows = kWaves * kWaveRows;

template <typename T>
constexpr int tile_rows() {
    return sizeof(T) == 4 ? 32 : 64;
}

// Gradients of scores, in float16, times a power of two that a column keeps to itself and
// lowers where a larger one comes: they may be of any size, and float16 has few.
struct Range {
    static constexpr float kFirst = 0x1p100f, kMost = 0x1p15f;
    float up = kFirst;

    template <int N>
    __device__ __forceinline__ void fit(f32x16 (&acc)[N], const f32x16& x) {
        float top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, __builtin_fabsf(x[i]));
        if (__any(top * up > kMost)) {
            const f32x2 tops = both_halves(top);
            top = fmaxf(tops[0], tops[1]);
            const float next = top * up > kMost ? __builtin_ldexpf(1.0f, 13 - __builtin_amdgcn_frexp_expf(top)) : up;
            const float f = next / up;  // powers of two
            up = next;
#pragma unroll
            for (int d = 0; d < N; ++d) acc[d] *= f;
        }
    }
};

// With p = exp(scale s - lse) and dp = dout v^T: ds = p (dp - delta), delta = dout . out of
// a row, and dq = scale ds k.  As the forward pass: a row's statistics are its lane's.
template <typename T, int D, bool Vec>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) * D > 256 ? 1 : 2) void attention_grad_q(AttentionGradArgs a) {
    constexpr int kKeys = tile_rows<T>(), kSteps = D / 16, kParts = D / 32;
    constexpr bool kHalf = __is_same(T, _Float16);
    constexpr uint32_t kBytes = kKeys * RowTile<T, D>::kPitch;
    __shared__ __align__(16) uint8_t k0[kBytes], v0[kBytes], k1[kBytes], v1[kBytes];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = lane & 31, h = lane >> 5;
    const uint32_t index = xcd_index(), head = index / a.pieces;
    const Piece piece = find_piece(a.offsets, a.wide_offsets, a.sequences, a.tokens, a.group, kRows, index % a.pieces, a.pieces);
    T* const dq = static_cast<T*>(a.dq);
    if (!piece.n) return clear_spare(piece, a.tokens, dq, a.dq_token, a.dq_head, head * a.group, a.group, a.dim);

    const uint32_t rows = piece.n * a.group;
    const uint32_t row0 = ((rows - 1) / kRows - piece.piece) * kRows, row1 = min(row0 + kRows, rows) - 1;
    const uint32_t t0 = row0 / a.group, t1 = row1 / a.group;
    const KeyList keys(t0, t1, a.window, a.sinks);
    const int32_t lo = (int32_t)keys.lo;
    const uint32_t wave_row = row0 + wave * kWaveRows, row = min(wave_row + c, rows - 1);
    const uint32_t token = row / a.group, q_head = head * a.group + row % a.group;
    const int32_t at = (int32_t)token - lo;
    const int32_t at0 = (int32_t)(min(wave_row, rows - 1) / a.group) - lo, at1 = (int32_t)(min(wave_row + 31, rows - 1) / a.group) - lo;
    const uint64_t packed = piece.first + token;
    Operand8<T> q[kSteps], dout[kSteps];
    // delta by the instructions that make dp, in their order: where a row sees one key, and
    // out is its value, ds is zero
    float delta = 0;
    {
        const T* p = static_cast<const T*>(a.q) + packed * a.q_token + q_head * a.q_head;
        const T* dp = static_cast<const T*>(a.dout) + packed * a.dout_token + q_head * a.dout_head;
        const T* o = static_cast<const T*>(a.out) + packed * a.out_token + q_head * a.out_head;
        f32x16 dots = {};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            q[s] = load8<T, Vec>(p, 16 * s + 8 * h, a.dim);
            dout[s] = load8<T, Vec>(dp, 16 * s + 8 * h, a.dim);
            dots = multiply(load8<T, Vec>(o, 16 * s + 8 * h, a.dim), dout[s], dots);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) delta = 8 * (i / 4) + 4 * h + i % 4 == c ? dots[i] : delta;
        const f32x2 both = both_halves(delta);  // zero in the half that has none
        delta = both[0] + both[1];
    }
    const float lse = a.lse[packed * a.heads + q_head] * kLog2e, scale = a.scale * kLog2e;
    if (h == 0 && wave_row + c < rows) {
        a.rows[packed * a.heads + q_head] = lse;
        a.rows[(uint64_t)a.tokens * a.heads + packed * a.heads + q_head] = delta;
    }

    const auto stage = [&](int32_t i0, uint8_t* k, uint8_t* v) SLLM_INLINE {
        const auto row_of = [&](const void* from, uint64_t token_stride, uint64_t head_stride, uint32_t r) SLLM_INLINE -> const T* {
            const int32_t i = i0 + (int32_t)r, n = i - keys.sinks;
            if (i >= keys.total) return nullptr;
            return static_cast<const T*>(from) + head * head_stride + (uint64_t)(piece.first + (uint32_t)(n < 0 ? i : lo + n)) * token_stride;
        };
        stage_rows<T, D, kKeys, kWaves, Vec>(k, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.k, a.k_token, a.k_head, r); });
        stage_rows<T, D, kKeys, kWaves, Vec>(v, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.v, a.v_token, a.v_head, r); });
    };
    f32x16 acc[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) acc[d] = f32x16{};
    Range range;
    const uint32_t rows_at = rows_from<T, D>(lane), columns_at = columns_from<T, D>(lane);
    const auto tile = [&](int32_t i0, const uint8_t* k, const uint8_t* v, auto masked) SLLM_INLINE {
        constexpr bool kMasked = decltype(masked)::value;
        const auto sees = [&](int r) SLLM_INLINE { return i0 + r < keys.total && keys.sees(at, i0 + r); };
        Operand8<T> ds[kKeys / 16];
#pragma unroll
        for (int n = 0; n < kKeys / 32; ++n) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s = multiply(read_rows<T, D>(k, rows_at, 32 * n, i), q[i], s);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) dp = multiply(read_rows<T, D>(v, rows_at, 32 * n, i), dout[i], dp);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -lse)) * (dp[i] - delta);
                if (kMasked && !sees(32 * n + 8 * (i / 4) + 4 * h + i % 4)) s[i] = 0;
            }
            if constexpr (kHalf) {
                const float before = range.up;
                range.fit(acc, s);
                if (n && __any(before != range.up)) {
                    // what this tile has rounded already was times the former power
                    const _Float16 f = (_Float16)(range.up / before);
#pragma unroll
                    for (int t = 0; t < 2 * n; ++t)
                        ds[t].v = __builtin_bit_cast(u32x4, __builtin_bit_cast(f16x8, ds[t].v) * f);
                }
                s *= range.up;
            }
            ds[2 * n] = as_operand<T>(s, 0);
            ds[2 * n + 1] = as_operand<T>(s, 1);
        }
        add_weighted<T, D, kKeys, kMasked>(acc, k, columns_at, 0, ds, sees);
    };
    const auto step = [&](int32_t i0, const uint8_t* k, const uint8_t* v, uint8_t* next_k, uint8_t* next_v) SLLM_INLINE {
        wait_but_loads<0>();
        barrier();
        if (i0 + kKeys < keys.total) stage(i0 + kKeys, next_k, next_v);
        if (keys.all(at0, at1, i0, i0 + kKeys - 1))
            tile(i0, k, v, std::false_type());
        else if (!keys.none(at0, at1, i0, i0 + kKeys - 1))
            tile(i0, k, v, std::true_type());
    };
    stage(0, k0, v0);
    for (int32_t i0 = 0; i0 < keys.total; i0 += 2 * kKeys) {
        step(i0, k0, v0, k1, v1);
        if (i0 + kKeys < keys.total) step(i0 + kKeys, k1, v1, k0, v0);
    }
    if (wave_row + c >= rows) return;
    store_column<T, D, Vec>(acc, kHalf ? a.scale / range.up : a.scale, dq + packed * a.dq_token + q_head * a.dq_head, a.dim);
}

// dv = p^T dout and dk = scale ds^T q, over the rows (tokens times heads that share the
// key) that see a key.  A wave has 32 keys, whose statistics are their lanes' own, and the
// rows come by; scores are of (rows x keys), their gradients' sums of (elements x keys).
template <typename T, int D, bool Vec>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) * D > 128 ? 1 : 2) void attention_grad_kv(AttentionGradArgs a) {
    constexpr int kTile = tile_rows<T>(), kSteps = D / 16, kParts = D / 32;
    constexpr bool kHalf = __is_same(T, _Float16);
    constexpr uint32_t kBytes = kTile * RowTile<T, D>::kPitch;
    __shared__ __align__(16) uint8_t q0[kBytes], o0[kBytes], q1[kBytes], o1[kBytes];
    __shared__ __align__(16) uint8_t l0[256], d0[256], l1[256], d1[256];  // rows' lse and delta
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = lane & 31, h = lane >> 5;
    const uint32_t index = xcd_index(), head = index / a.pieces;
    const Piece piece = find_piece(a.offsets, a.wide_offsets, a.sequences, a.tokens, 1, kRows, index % a.pieces, a.pieces);
    T *const dk = static_cast<T*>(a.dk), *const dv = static_cast<T*>(a.dv);
    if (!piece.n) {
        clear_spare(piece, a.tokens, dk, a.dk_token, a.dk_head, head, 1, a.dim);
        clear_spare(piece, a.tokens, dv, a.dv_token, a.dv_head, head, 1, a.dim);
        return;
    }
    const uint32_t window = a.window, sinks = a.sinks;
    const uint32_t key0 = piece.piece * kRows, key1 = min(key0 + kRows, piece.n) - 1;
    const uint32_t last = key0 < sinks ? piece.n - 1 : min(piece.n - 1, key1 + window - 1);  // the last token that sees one
    const uint32_t row_first = key0 * a.group, row_end = (last + 1) * a.group;
    const uint32_t wave_key0 = min(key0 + wave * kWaveRows, key1), wave_key1 = min(wave_key0 + kWaveRows - 1, key1);
    const uint32_t key = min(key0 + wave * kWaveRows + c, key1);
    Operand8<T> k[kSteps], v[kSteps];
    {
        const T* p = static_cast<const T*>(a.k) + (uint64_t)(piece.first + key) * a.k_token + head * a.k_head;
        const T* pv = static_cast<const T*>(a.v) + (uint64_t)(piece.first + key) * a.v_token + head * a.v_head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            k[s] = load8<T, Vec>(p, 16 * s + 8 * h, a.dim);
            v[s] = load8<T, Vec>(pv, 16 * s + 8 * h, a.dim);
        }
    }
    const auto stage = [&](uint32_t r0, uint8_t* q, uint8_t* dout, uint8_t* lse, uint8_t* delta) SLLM_INLINE {
        const auto row_of = [&](const void* from, uint64_t token_stride, uint64_t head_stride, uint32_t r) SLLM_INLINE -> const T* {
            const uint32_t row = r0 + r, token = row / a.group;
            if (row >= row_end) return nullptr;
            return static_cast<const T*>(from) + (uint64_t)(piece.first + token) * token_stride + (head * a.group + row - token * a.group) * head_stride;
        };
        stage_rows<T, D, kTile, kWaves, Vec>(q, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.q, a.q_token, a.q_head, r); });
        stage_rows<T, D, kTile, kWaves, Vec>(dout, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.dout, a.dout_token, a.dout_head, r); });
        if (wave < 2) {
            const uint32_t row = min(r0 + lane % kTile, row_end - 1), token = row / a.group;
            const float* p = a.rows + (wave ? (uint64_t)a.tokens * a.heads : 0);
            load_word_to_lds(p + (uint64_t)(piece.first + token) * a.heads + head * a.group + row - token * a.group, wave ? delta : lse, 0);
        }
    };
    // p is times 2^kUp, which makes float16's least of them normal numbers, and so is ds
    constexpr float kUp = kHalf ? 15.0f : 0.0f;
    const float scale = a.scale * kLog2e;
    f32x16 acc_k[kParts], acc_v[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) acc_k[d] = acc_v[d] = f32x16{};
    Range range;
    const uint32_t rows_at = rows_from<T, D>(lane), columns_at = columns_from<T, D>(lane);
    const auto tile = [&](uint32_t r0, const uint8_t* q, const uint8_t* dout, const uint8_t* lse, const uint8_t* delta, auto masked) SLLM_INLINE {
        constexpr bool kMasked = decltype(masked)::value;
        const auto sees = [&](int r) SLLM_INLINE {
            const uint32_t row = r0 + (uint32_t)r, token = row / a.group;
            return row < row_end && token >= key && (token - key < window || key < sinks);
        };
#pragma unroll 1
        for (int n = 0; n < kTile / 32; ++n) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s = multiply(read_rows<T, D>(q, rows_at, 32 * n, i), k[i], s);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) dp = multiply(read_rows<T, D>(dout, rows_at, 32 * n, i), v[i], dp);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 l = lds_read<f32x4>(lse, h * 16 + (32 * n + 8 * g) * 4), de = lds_read<f32x4>(delta, h * 16 + (32 * n + 8 * g) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + i], scale, kUp - l[i]));
                    float d = p * (dp[4 * g + i] - de[i]);
                    if (kMasked && !sees(32 * n + 8 * g + 4 * h + i)) p = d = 0;
                    s[4 * g + i] = p, dp[4 * g + i] = d;
                }
            }
            const Operand8<T> p[2] = {as_operand<T>(s, 0), as_operand<T>(s, 1)};
            add_weighted<T, D, 32, kMasked>(acc_v, dout, columns_at, 32 * n, p, sees);
            if constexpr (kHalf) {
                range.fit(acc_k, dp);
                dp *= range.up;
            }
            const Operand8<T> ds[2] = {as_operand<T>(dp, 0), as_operand<T>(dp, 1)};
            add_weighted<T, D, 32, kMasked>(acc_k, q, columns_at, 32 * n, ds, sees);
        }
    };
    const auto step = [&](uint32_t r0, const uint8_t* q, const uint8_t* o, const uint8_t* l, const uint8_t* d, uint8_t* next_q, uint8_t* next_o,
                          uint8_t* next_l, uint8_t* next_d) SLLM_INLINE {
        wait_but_loads<0>();
        barrier();
        if (r0 + kTile < row_end) stage(r0 + kTile, next_q, next_o, next_l, next_d);
        const uint32_t qa = r0 / a.group, qb = min(r0 + kTile, row_end) - 1, ta = qa, tb = qb / a.group;
        if (ta >= wave_key1 && r0 + kTile <= row_end && (tb - wave_key0 < window || wave_key1 < sinks))
            tile(r0, q, o, l, d, std::false_type());
        else if (!(tb < wave_key0 || (wave_key0 >= sinks && ta >= wave_key1 + window)))
            tile(r0, q, o, l, d, std::true_type());
    };
    stage(row_first, q0, o0, l0, d0);
    for (uint32_t r0 = row_first; r0 < row_end; r0 += 2 * kTile) {
        step(r0, q0, o0, l0, d0, q1, o1, l1, d1);
        if (r0 + kTile < row_end) step(r0 + kTile, q1, o1, l1, d1, q0, o0, l0, d0);
    }
    if (key0 + wave * kWaveRows + c > key1) return;
    const uint64_t packed = piece.first + key;
    store_column<T, D, Vec>(acc_v, kHalf ? 0x1p-15f : 1.0f, dv + packed * a.dv_token + head * a.dv_head, a.dim);
    store_column<T, D, Vec>(acc_k, kHalf ? a.scale * 0x1p-15f / range.up : a.scale, dk + packed * a.dk_token + head * a.dk_head, a.dim);
}

template <typename T, int D>
void launch(AttentionGradArgs a, hipStream_t stream) {
    const uint32_t more = a.offsets ? a.sequences : 0;
    a.pieces = (uint32_t)ceil_div((uint64_t)a.tokens * a.group, kRows) + more;
    (a.vec ? attention_grad_q<T, D, true> : attention_grad_q<T, D, false>)<<<dim3(a.pieces * a.kv_heads), kWaves * 64, 0, stream>>>(a);
    a.pieces = (uint32_t)ceil_div(a.tokens, kRows) + more;
    (a.vec ? attention_grad_kv<T, D, true> : attention_grad_kv<T, D, false>)<<<dim3(a.pieces * a.kv_heads), kWaves * 64, 0, stream>>>(a);
}

}  // namespace

uint64_t attention_grad_workspace(const AttentionArgs& a) { return (uint64_t)a.tokens * a.heads * 8; }

int32_t launch_attention_grad(AttentionGradArgs a, void* workspace, hipStream_t stream) {
    a.rows = static_cast<float*>(workspace);
    SLLM_BY_DTYPE(a.dtype, T, {
        if (a.dim <= 64)
            launch<T, 64>(a, stream);
        else
            launch<T, 128>(a, stream);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
