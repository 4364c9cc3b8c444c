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

// A logarithm of a row's sum past this, to the base of two, is not enough to tell the row's weights:
// in 32 bits, rounded four times on its way, it is off by up to 2^-22 of itself, and so are
// they.  Such rows' largest score and the sum against it are found again, one product more (32 heads
// of 128 elements, 8192 tokens in four sequences, a window of 1024, bf16, every row so: 700 us and 797;
// rows that are not pay 1 % for the choice).
constexpr float kFar = 0x1p9f;

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

// With p = exp(scale s - lse), rows far from zero apart, and dp = dout v^T: ds = p (dp - delta), delta = dout . out of
// a row, and dq = scale ds k.  As the forward pass: a row's statistics are its lane's.
//
// Three products of a tile, one of them twice, since ds is rounded: 32 heads of 128 elements,
// 8192 tokens in four sequences, a window of 1024, bf16: 314 to 344 us, the matrix cores busy 34 %
// of the cycles, the vector units 31 %.  2176 workgroups at two a CU are 4.25 rounds, of which each
// workgroup starts with a wait for its first tiles and the last has three places in four
// empty: 1.6 waves a SIMD.
template <typename T, int D, bool Vec>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) * D > 256 ? 1 : 2) void attention_grad_q(AttentionGradArgs a) {
    constexpr int kKeys = tile_rows<T>(), kSteps = D / 16, kParts = D / 32;
    constexpr bool kHalf = __is_same(T, _Float16), kTwice = sizeof(T) == 2;
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
    const KeyList::Sight sight = keys.sight((int32_t)token - lo);
    const int32_t at0 = (int32_t)(min(wave_row, rows - 1) / a.group) - lo, at1 = (int32_t)(min(wave_row + 31, rows - 1) / a.group) - lo;
    const uint64_t packed = piece.first + token;
    Operand8<T> q[kSteps], dout[kSteps];
    const float scale = a.scale * kLog2e;
    float lse = a.lse[packed * a.heads + q_head] * kLog2e, less = 0;  // p = 2^(scale (s - less) - lse)
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
    const bool far = __builtin_fabsf(lse) > kFar && __builtin_fabsf(lse) < __builtin_inff();
    __shared__ uint32_t wave_far[kWaves];
    const uint32_t some_far = __any(far);
    if (lane == 0) wave_far[wave] = some_far;
    __syncthreads();
    static_assert(kWaves == 4, "");
    const bool any_far = __builtin_amdgcn_readfirstlane(wave_far[0] | wave_far[1] | wave_far[2] | wave_far[3]);

    const bool repeats = Vec && a.dim == D && max(a.k_token, a.v_token) < (1u << 24);
    LaneOffsets<T, D, kKeys, kWaves> k_at, v_at;
    if constexpr (Vec) {
        k_at.set(k_at.kRun * a.k_token, [&](uint32_t r) SLLM_INLINE { return r * (uint32_t)a.k_token; });
        v_at.set(v_at.kRun * a.v_token, [&](uint32_t r) SLLM_INLINE { return r * (uint32_t)a.v_token; });
    }
    const auto stage = [&](int32_t i0, uint8_t* k, uint8_t* v) SLLM_INLINE {
        if (repeats && i0 >= keys.sinks && i0 + kKeys <= keys.total) {
            const uint64_t token = piece.first + (uint32_t)(lo + i0 - keys.sinks);
            k_at.stage(k, static_cast<const T*>(a.k) + head * a.k_head + token * a.k_token);
            v_at.stage(v, static_cast<const T*>(a.v) + head * a.v_head + token * a.v_token);
            return;
        }
        const auto row_of = [&](const void* from, uint64_t token_stride, uint64_t head_stride, uint32_t r) SLLM_INLINE -> const T* {
            const int32_t i = min(i0 + (int32_t)r, keys.total - 1), n = i - keys.sinks;
            const T* p = static_cast<const T*>(from) + head * head_stride + (uint64_t)(piece.first + (uint32_t)(n < 0 ? i : lo + n)) * token_stride;
            return i0 + (int32_t)r < keys.total ? p : nullptr;
        };
        stage_rows<T, D, kKeys, kWaves, Vec>(k, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.k, a.k_token, a.k_head, r); });
        stage_rows<T, D, kKeys, kWaves, Vec>(v, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.v, a.v_token, a.v_head, r); });
    };
    const auto each_tile = [&](const auto& work) SLLM_INLINE {
        const auto step = [&](int32_t i0, const uint8_t* k, const uint8_t* v, uint8_t* next_k, uint8_t* next_v) SLLM_INLINE {
            wait_but_loads<0>();
            barrier();
            if (i0 + kKeys < keys.total) stage(i0 + kKeys, next_k, next_v);
            if (!keys.none(at0, at1, i0, i0 + kKeys - 1)) work(i0, k, v, !keys.all(at0, at1, i0, i0 + kKeys - 1));
        };
        stage(0, k0, v0);
        for (int32_t i0 = 0; i0 < keys.total; i0 += 2 * kKeys) {
            step(i0, k0, v0, k1, v1);
            if (i0 + kKeys < keys.total) step(i0 + kKeys, k1, v1, k0, v0);
        }
    };
    const uint32_t rows_at = rows_from<T, D>(lane), columns_at = columns_from<T, D>(lane);
    if (any_far) {
        Reference<float> ref;
        float sum = 0;
        each_tile([&](int32_t i0, const uint8_t* k, const uint8_t*, bool masked) SLLM_INLINE {
#pragma unroll
            for (int n = 0; n < kKeys / 32; ++n) {
                RowFragments<T, D> f;
                f.read(k, rows_at, 32 * n);
                f32x16 s = f.times(q);
                if (masked) {
                    const KeyList::Sight here = sight.here();
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = here.sees(i0 + 32 * n + 8 * (i / 4) + 4 * (int32_t)h + i % 4) ? s[i] : -__builtin_inff();
                }
                float top = s[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
                const f32x2 tops = both_halves(top);
                sum *= ref.raise(fmaxf(ref.most, fmaxf(tops[0], tops[1])), scale);
                const float finite = ref.finite();
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += ref.weight(s[i], scale, finite);
            }
        });
        const f32x2 sums = both_halves(sum);
        if (far) less = ref.most, lse = __builtin_amdgcn_logf(sums[0] + sums[1]);
        wait_but_loads<0>();
        barrier();  // the tiles have been read
    }
    const auto weigh = [&](f32x16& s, const f32x16& dp, int32_t i0, bool masked, auto any_less) SLLM_INLINE {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float near = decltype(any_less)::value ? s[i] - less : s[i];
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(near, scale, -lse)) * (dp[i] - delta);
        }
        if (masked) {
            const KeyList::Sight here = sight.here();
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = here.sees(i0 + 8 * (i / 4) + 4 * (int32_t)h + i % 4) ? s[i] : 0.0f;
        }
    };
    // A row's ds sum to zero.  What they do sum to, delta is off by: out has been rounded, and
    // its weights.  Of many keys that is little; where there are few they are gone through once
    // for it.  (Of two bf16 keys dq is off by 0.0043 of itself without, 0.0017 with; of some ten
    // by a third more than with.)
    constexpr int32_t kFew = 3 * 64;
    if (kTwice && keys.total <= kFew) {
        float sum = 0;
        each_tile([&](int32_t i0, const uint8_t* k, const uint8_t* v, bool masked) SLLM_INLINE {
#pragma unroll
            for (int n = 0; n < kKeys / 32; ++n) {
                RowFragments<T, D> f;
                f.read(k, rows_at, 32 * n);
                f32x16 s = f.times(q);
                f.read(v, rows_at, 32 * n);
                weigh(s, f.times(dout), i0 + 32 * n, masked, std::true_type());
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += s[i];
            }
        });
        const f32x2 sums = both_halves(sum);
        delta += sums[0] + sums[1];
        wait_but_loads<0>();
        barrier();  // the tiles have been read
    }
    if (h == 0 && wave_row + c < rows) {
        a.rows[packed * a.heads + q_head] = lse;
        a.rows[(uint64_t)a.tokens * a.heads + packed * a.heads + q_head] = delta;
        a.rows[(uint64_t)a.tokens * a.heads * 2 + packed * a.heads + q_head] = less;
    }

    f32x16 acc[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) acc[d] = f32x16{};
    Range range;
    bool out_of_sight = false;  // something was taken out
    const auto tile = [&](int32_t i0, const uint8_t* k, const uint8_t* v, bool masked, auto any_less) SLLM_INLINE {
        RowFragments<T, D> kf, vf;
        ColumnFragments<T, D, 32> cf;
        const bool bad = masked && any_not_finite<T, D, kKeys>(k);
        out_of_sight |= bad;
        kf.read(k, rows_at, 0);
#pragma unroll
        for (int n = 0; n < kKeys / 32; ++n) {
            phase();
            vf.read(v, rows_at, 32 * n);
            f32x16 s = kf.times(q);
            phase();
            cf.read(k, columns_at, 32 * n, 0);
            const f32x16 dp = vf.times(dout);
            phase();
            weigh(s, dp, i0 + 32 * n, masked, any_less);
            if constexpr (kHalf) {
                range.fit(acc, s);
                s *= range.up;
            }
            const Operand8<T> ds[2] = {as_operand<T>(s, 0), as_operand<T>(s, 1)};
            Operand8<T> rest[2];
            if constexpr (kTwice) {
                const f32x16 r = rounded_off<T>(s, ds);
                rest[0] = as_operand<T>(r, 0), rest[1] = as_operand<T>(r, 1);
            }
            phase();
            if (n + 1 < kKeys / 32) kf.read(k, rows_at, 32 * (n + 1));
#pragma unroll
            for (int d = 0; d < kParts; ++d) {
                ColumnFragments<T, D, 32> next;
                if (d + 1 < kParts) next.read(k, columns_at, 32 * n, d + 1);
                if (bad) cf.take_out();
                cf.add(acc[d], ds);
                if constexpr (kTwice) cf.add(acc[d], rest);
                phase();
                if (d + 1 < kParts) cf = next;
            }
        }
    };
    // (two loops: to take `less` from all scores costs 3 % where it is zero)
    if (any_far)
        each_tile([&](int32_t i0, const uint8_t* k, const uint8_t* v, bool masked) SLLM_INLINE { tile(i0, k, v, masked, std::true_type()); });
    else
        each_tile([&](int32_t i0, const uint8_t* k, const uint8_t* v, bool masked) SLLM_INLINE { tile(i0, k, v, masked, std::false_type()); });
    if (out_of_sight)
        for (int32_t i = 0; i < keys.total; ++i)
            put_back<T, D>(acc, static_cast<const T*>(a.k) + head * a.k_head + (uint64_t)(piece.first + (uint32_t)(i < keys.sinks ? i : lo + i - keys.sinks)) * a.k_token,
                           a.dim, sight.sees(i));
    if (wave_row + c >= rows) return;
    store_column<T, D, Vec>(acc, kHalf ? a.scale / range.up : a.scale, dq + packed * a.dq_token + q_head * a.dq_head, a.dim);
}

// Tile `index` of the keys that are sinks; none: n = 0.
__device__ __forceinline__ Piece find_sinks(const AttentionGradArgs& a, uint32_t index) {
    Piece p;
    if (a.sink_tiles) {  // one sequence after the other
        p = {index / a.sink_tiles, 0, 0, index % a.sink_tiles, 1, 0};
        find_sequence(a.offsets, a.wide_offsets, p.sequence, a.tokens, p.first, p.n);
    } else {
        p = find_piece(a.offsets, a.wide_offsets, a.sequences, a.tokens, 1, kRows, index, a.pieces);
    }
    if (p.piece * kRows >= min(p.n, (uint32_t)a.sinks)) p.n = 0;
    return p;
}

// Where part s of a sink's sums is, by its place among the tokens or by sequence.
__device__ __forceinline__ uint64_t far_at(const AttentionGradArgs& a, uint32_t s, const Piece& p, uint32_t key, uint32_t head) {
    const uint64_t row = a.far_packed ? (uint64_t)p.first + key : (uint64_t)p.sequence * a.sinks + key;
    return ((2 * s * a.far_rows + row) * a.kv_heads + head) * a.dim;
}

// dv = p^T dout and dk = scale ds^T q, over the rows (tokens times heads that share the
// key) that see a key.  A wave has 32 keys, whose statistics are their lanes' own, and the
// rows come by; scores are of (rows x keys), their gradients' sums of (elements x keys).
//
// Two waves of a SIMD hide each other's waits: for that a wave has its keys and the sums in
// registers, but takes its values from LDS each time (with 512 registers and one wave a SIMD
// 587 us, so 480 in that form).  Four products of a tile, one of them twice; the same texts take 381 to 412
// us, the matrix cores busy 32 % of the cycles, the vector units 33 %, LDS 20 %.
//
// Far: what the rows behind the window give to the sinks of a tile, every row of a long text
// to a few keys.  That is split over many workgroups and joined afterwards.  (Left to the tiles
// of the sinks, a text of 8192 tokens in 32 heads that share 8 heads of keys, a window of 1024
// and four sinks took 3.4 ms, without sinks 0.92.)
template <typename T, int D, bool Vec, bool Far>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) * D > 256 ? 1 : 2) void attention_grad_kv(AttentionGradArgs a) {
    constexpr int kTile = 32, kSteps = D / 16, kParts = D / 32;
    constexpr bool kHalf = __is_same(T, _Float16), kTwice = sizeof(T) == 2;
    constexpr uint32_t kBytes = kTile * RowTile<T, D>::kPitch;
    __shared__ __align__(16) uint8_t q0[kBytes], o0[kBytes], q1[kBytes], o1[kBytes];
    __shared__ __align__(16) uint8_t l0[256], d0[256], e0[256], l1[256], d1[256], e1[256];  // rows' lse, delta and less
    __shared__ __align__(16) uint8_t values[kRows * RowTile<T, D>::kPitch];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = lane & 31, h = lane >> 5;
    const uint32_t splits = Far ? a.far : a.splits, index = Far ? blockIdx.x : xcd_index(), split = index % splits;
    const uint32_t head = index / splits / a.pieces;
    const Piece piece = Far ? find_sinks(a, index / splits % a.pieces)
                            : find_piece(a.offsets, a.wide_offsets, a.sequences, a.tokens, 1, kRows, index / splits % a.pieces, a.pieces);
    if (Far && !piece.n) return;
    T *const dk = static_cast<T*>(a.dk), *const dv = static_cast<T*>(a.dv);
    // sums of a part of the rows, to be joined: of this split, keys and then values
    const uint64_t part_token = (uint64_t)a.kv_heads * a.dim, part_size = a.tokens * part_token;
    float *const part_k = a.parts + 2 * split * part_size, *const part_v = part_k + part_size;
    if (!piece.n) {
        if (a.splits > 1) {
            clear_spare(piece, a.tokens, part_k, part_token, a.dim, head, 1, a.dim);
            clear_spare(piece, a.tokens, part_v, part_token, a.dim, head, 1, a.dim);
        } else {
            clear_spare(piece, a.tokens, dk, a.dk_token, a.dk_head, head, 1, a.dim);
            clear_spare(piece, a.tokens, dv, a.dv_token, a.dv_head, head, 1, a.dim);
        }
        return;
    }
    const uint32_t window = a.window, sinks = a.sinks;
    const uint32_t key0 = piece.piece * kRows, key1 = min(key0 + kRows, piece.n) - 1;
    const uint32_t near_end = min(piece.n, key1 + window);  // behind the last token whose window holds one
    const uint32_t all_first = (Far ? near_end : key0) * a.group, all_end = (Far ? piece.n : near_end) * a.group;
    // this split's rows, whole tiles of them, perhaps none
    const uint32_t share = ((all_end - all_first + kTile - 1) / kTile + splits - 1) / splits * kTile;
    const uint32_t row_first = min(all_first + split * share, all_end), row_end = min(row_first + share, all_end);
    const uint32_t wave_key0 = min(key0 + wave * kWaveRows, key1), wave_key1 = min(wave_key0 + kWaveRows - 1, key1);
    const uint32_t key = min(key0 + wave * kWaveRows + c, key1);
    // the rows that see a key
    const auto seen_rows = [&](uint32_t key, uint32_t& from, uint32_t& n) SLLM_INLINE {
        from = key * a.group;
        n = (key < sinks ? piece.n - key : min(piece.n - key, window)) * a.group;
    };
    Operand8<T> k[kSteps];
    {
        const T* p = static_cast<const T*>(a.k) + (uint64_t)(piece.first + key) * a.k_token + head * a.k_head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) k[s] = load8<T, Vec>(p, 16 * s + 8 * h, a.dim);
    }
    stage_rows<T, D, kRows, kWaves, Vec>(values, a.dim, [&](uint32_t r) SLLM_INLINE -> const T* {
        return static_cast<const T*>(a.v) + (uint64_t)(piece.first + min(key0 + r, key1)) * a.v_token + head * a.v_head;
    });
    // Tiles whose rows lie alike, a whole number of tokens each, need no look at each.
    typedef LaneOffsets<T, D, kTile, kWaves> Offsets;
    const bool repeats = Vec && a.dim == D && Offsets::kRun % a.group == 0 && max(max(a.q_token, a.dout_token), max(a.q_head, a.dout_head)) < (1u << 24);
    Offsets q_at, o_at;
    if constexpr (Vec) {
        const uint32_t tokens = Offsets::kRun / a.group;
        const auto place = [&](uint64_t token_stride, uint64_t head_stride, uint32_t r) SLLM_INLINE {
            return r / a.group * (uint32_t)token_stride + r % a.group * (uint32_t)head_stride;
        };
        q_at.set(tokens * a.q_token, [&](uint32_t r) SLLM_INLINE { return place(a.q_token, a.q_head, r); });
        o_at.set(tokens * a.dout_token, [&](uint32_t r) SLLM_INLINE { return place(a.dout_token, a.dout_head, r); });
    }
    const uint32_t heads0 = head * a.group;
    const auto stage = [&](uint32_t r0, uint8_t* q, uint8_t* dout, uint8_t* lse, uint8_t* delta, uint8_t* less) SLLM_INLINE {
        if (wave < 3) {
            const uint32_t row = min(r0 + lane % kTile, row_end - 1), token = row / a.group;
            const float* p = a.rows + wave * (uint64_t)a.tokens * a.heads;
            load_word_to_lds(p + (uint64_t)(piece.first + token) * a.heads + heads0 + row - token * a.group, wave == 0 ? lse : wave == 1 ? delta : less, 0);
        }
        if (repeats && r0 + kTile <= row_end) {
            const uint64_t token = piece.first + r0 / a.group;
            q_at.stage(q, static_cast<const T*>(a.q) + token * a.q_token + heads0 * a.q_head);
            o_at.stage(dout, static_cast<const T*>(a.dout) + token * a.dout_token + heads0 * a.dout_head);
            return;
        }
        const auto row_of = [&](const void* from, uint64_t token_stride, uint64_t head_stride, uint32_t r) SLLM_INLINE -> const T* {
            const uint32_t row = min(r0 + r, row_end - 1), token = row / a.group;
            const T* p = static_cast<const T*>(from) + (uint64_t)(piece.first + token) * token_stride + (heads0 + row - token * a.group) * head_stride;
            return r0 + r < row_end ? p : nullptr;
        };
        stage_rows<T, D, kTile, kWaves, Vec>(q, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.q, a.q_token, a.q_head, r); });
        stage_rows<T, D, kTile, kWaves, Vec>(dout, a.dim, [&](uint32_t r) SLLM_INLINE { return row_of(a.dout, a.dout_token, a.dout_head, r); });
    };
    // p is times 2^kUp, which makes float16's least of them normal numbers, and so is ds
    constexpr float kUp = kHalf ? 15.0f : 0.0f;
    const float scale = a.scale * kLog2e;
    f32x16 acc_k[kParts], acc_v[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) acc_k[d] = acc_v[d] = f32x16{};
    Range range;
    bool out_of_sight = false;  // something was taken out
    const auto tile = [&](uint32_t r0, const uint8_t* q, const uint8_t* dout, const uint8_t* lse, const uint8_t* delta, const uint8_t* less,
                          bool masked) SLLM_INLINE {
        // places of fragments are made anew each time: kept, they would take what sums need
        uint32_t here = threadIdx.x;
        asm volatile("" : "+v"(here));
        const uint32_t rows_at = rows_from<T, D>(here & 63), columns_at = columns_from<T, D>(here & 63), h = here >> 5 & 1;
        const uint32_t values_at = rows_at + wave * kWaveRows * RowTile<T, D>::kPitch;
        // two steps of both products at a time, their fragments read a run ahead
        struct Run {
            Operand8<T> q[2], o[2], v[2];
        };
        const auto read = [&](Run& f, int i) SLLM_INLINE {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f.q[j] = read_rows<T, D>(q, rows_at, 0, i + j);
                f.o[j] = read_rows<T, D>(dout, rows_at, 0, i + j);
                f.v[j] = read_rows<T, D>(values, values_at, 0, i + j);
            }
        };
        bool bad = false;
        f32x16 s = {}, dp = {};
        Run run;
        ColumnFragments<T, D, 32> oc, qc;
        const float one_less = lds_read<float>(less, (here & 31) * 4);
        read(run, 0);
        const bool some_far = __any(one_less != 0);
        __builtin_amdgcn_s_setprio(1);
        phase();
#pragma unroll
        for (int i = 0; i < kSteps; i += 2) {
            Run next;
            if (i + 2 < kSteps) {
                read(next, i + 2);
            } else {
                oc.read(dout, columns_at, 0, 0);
                qc.read(q, columns_at, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s = multiply(run.q[j], k[i + j], s);
                dp = multiply(run.o[j], run.v[j], dp);
            }
            phase();
            if (i + 2 < kSteps) run = next;
        }
        __builtin_amdgcn_s_setprio(0);
        if (some_far)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 e = lds_read<f32x4>(less, h * 16 + 8 * g * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * g + i] -= e[i];
            }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 l = lds_read<f32x4>(lse, h * 16 + 8 * g * 4), de = lds_read<f32x4>(delta, h * 16 + 8 * g * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[4 * g + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + i], scale, kUp - l[i]));
                dp[4 * g + i] = s[4 * g + i] * (dp[4 * g + i] - de[i]);
            }
        }
        if (masked) {
            uint32_t at = key0 + wave * kWaveRows + (here & 31);
            asm volatile("" : "+v"(at));  // not to be found out before this is reached
            uint32_t from, n_seen;
            seen_rows(min(at, key1), from, n_seen);
            n_seen = min(n_seen, max(row_end, from) - from);  // rows past the end have another's statistics
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool seen = r0 + 8 * (i / 4) + 4 * h + i % 4 - from < n_seen;
                s[i] = seen ? s[i] : 0.0f, dp[i] = seen ? dp[i] : 0.0f;
            }
            if constexpr (!Far) {  // (far rows are seen, or zeros)
                bad = any_not_finite<T, D, kTile>(dout) | any_not_finite<T, D, kTile>(q);
                out_of_sight |= bad;
            }
        }
        if constexpr (kHalf) {
            range.fit(acc_k, dp);
            dp *= range.up;
        }
        const Operand8<T> p[2] = {as_operand<T>(s, 0), as_operand<T>(s, 1)}, ds[2] = {as_operand<T>(dp, 0), as_operand<T>(dp, 1)};
        Operand8<T> rest[2];
        if constexpr (kTwice) {
            const f32x16 r = rounded_off<T>(dp, ds);
            rest[0] = as_operand<T>(r, 0), rest[1] = as_operand<T>(r, 1);
        }
        phase();
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int d = 0; d < kParts; ++d) {
            ColumnFragments<T, D, 32> next_o, next_q;
            if (d + 1 < kParts) {
                next_o.read(dout, columns_at, 0, d + 1);
                next_q.read(q, columns_at, 0, d + 1);
            }
            if (bad) {
                oc.take_out();
                qc.take_out();
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                acc_v[d] = multiply(oc.f[t], p[t], acc_v[d]);
                acc_k[d] = multiply(qc.f[t], ds[t], acc_k[d]);
            }
            if constexpr (kTwice) qc.add(acc_k[d], rest);
            phase();
            if (d + 1 < kParts) oc = next_o, qc = next_q;
        }
        __builtin_amdgcn_s_setprio(0);
    };
    const auto step = [&](uint32_t r0, const uint8_t* q, const uint8_t* o, const uint8_t* l, const uint8_t* d, const uint8_t* e, uint8_t* next_q,
                          uint8_t* next_o, uint8_t* next_l, uint8_t* next_d, uint8_t* next_e) SLLM_INLINE {
        wait_but_loads<0>();
        barrier();
        if (r0 + kTile < row_end) stage(r0 + kTile, next_q, next_o, next_l, next_d, next_e);
        if constexpr (Far) {
            // every sink is seen, and other keys' sums are not kept
            if (wave_key0 < sinks) tile(r0, q, o, l, d, e, r0 + kTile > row_end);
            return;
        }
        const uint32_t ta = r0 / a.group, tb = (min(r0 + kTile, row_end) - 1) / a.group;
        const bool all = ta >= wave_key1 && r0 + kTile <= row_end && (tb - wave_key0 < window || wave_key1 < sinks);
        if (!(tb < wave_key0 || (wave_key0 >= sinks && ta >= wave_key1 + window))) tile(r0, q, o, l, d, e, !all);
    };
    if (row_first < row_end)
        stage(row_first, q0, o0, l0, d0, e0);
    else
        wait_but_loads<0>();  // those of the values
    for (uint32_t r0 = row_first; r0 < row_end; r0 += 2 * kTile) {
        step(r0, q0, o0, l0, d0, e0, q1, o1, l1, d1, e1);
        if (r0 + kTile < row_end) step(r0 + kTile, q1, o1, l1, d1, e1, q0, o0, l0, d0, e0);
    }
    if (out_of_sight) {
        uint32_t seen_from, n_seen;
        seen_rows(key, seen_from, n_seen);
        for (uint32_t row = row_first; row < row_end; ++row) {
            const uint32_t token = row / a.group, q_head = heads0 + row % a.group;
            const bool seen = row - seen_from < n_seen;
            put_back<T, D>(acc_v, static_cast<const T*>(a.dout) + (uint64_t)(piece.first + token) * a.dout_token + q_head * a.dout_head, a.dim, seen);
            put_back<T, D>(acc_k, static_cast<const T*>(a.q) + (uint64_t)(piece.first + token) * a.q_token + q_head * a.q_head, a.dim, seen);
        }
    }
    if (key0 + wave * kWaveRows + c > key1) return;
    const uint64_t packed = piece.first + key;
    const float f_v = kHalf ? 0x1p-15f : 1.0f, f_k = kHalf ? a.scale * 0x1p-15f / range.up : a.scale;
    if (Far || (a.far && a.splits == 1 && key < sinks)) {
        // a part of a sink's sums: of the far rows' splits one after the other, then of the others
        if (key >= sinks) return;
        float* const to = a.far_parts + far_at(a, Far ? split : a.far, piece, key, head);
        store_column<float, D, Vec>(acc_k, f_k, to, a.dim);
        store_column<float, D, Vec>(acc_v, f_v, to + a.far_rows * a.kv_heads * a.dim, a.dim);
        return;
    }
    if (a.splits > 1) {
        store_column<float, D, Vec>(acc_v, f_v, part_v + packed * part_token + head * a.dim, a.dim);
        store_column<float, D, Vec>(acc_k, f_k, part_k + packed * part_token + head * a.dim, a.dim);
        return;
    }
    store_column<T, D, Vec>(acc_v, f_v, dv + packed * a.dv_token + head * a.dv_head, a.dim);
    store_column<T, D, Vec>(acc_k, f_k, dk + packed * a.dk_token + head * a.dk_head, a.dim);
}

// The splits' sums, first to last, so that every call adds in the same order (1333 tokens of 5
// heads of 80 elements, five splits: 8 us, reads that follow one another).
template <typename T>
__global__ __launch_bounds__(256) void join_kv(AttentionGradArgs a) {
    const uint64_t n = (uint64_t)a.tokens * a.kv_heads * a.dim, i = (uint64_t)block_index() * 256 + threadIdx.x;
    if (i >= n) return;
    float k = 0, v = 0;
    for (uint32_t s = 0; s < a.splits; ++s) k += a.parts[2 * s * n + i], v += a.parts[(2 * s + 1) * n + i];
    const uint64_t token = i / (a.kv_heads * a.dim);
    const uint32_t head = i / a.dim % a.kv_heads, e = i % a.dim;
    static_cast<T*>(a.dk)[token * a.dk_token + head * a.dk_head + e] = from_f32<T>(k);
    static_cast<T*>(a.dv)[token * a.dv_token + head * a.dv_head + e] = from_f32<T>(v);
}

// A sink's parts, in their order (4 sinks of 4 sequences in 32 heads, three parts: 5 us, a launch).
template <typename T>
__global__ __launch_bounds__(256) void join_sinks(AttentionGradArgs a) {
    const uint32_t head = blockIdx.x / a.pieces;
    const Piece piece = find_sinks(a, blockIdx.x % a.pieces);
    if (!piece.n) return;
    const uint32_t key0 = piece.piece * kRows, keys = min((uint32_t)kRows, min(piece.n, (uint32_t)a.sinks) - key0);
    const uint64_t size = (uint64_t)a.tokens * a.kv_heads * a.dim, values = a.far_rows * a.kv_heads * a.dim;
    for (uint32_t i = threadIdx.x; i < keys * a.dim; i += 256) {
        const uint32_t key = key0 + i / a.dim, e = i % a.dim;
        const uint64_t token = piece.first + key, at = (token * a.kv_heads + head) * a.dim + e;
        float k = 0, v = 0;
        if (a.splits > 1)
            for (uint32_t s = 0; s < a.splits; ++s) k += a.parts[2 * s * size + at], v += a.parts[(2 * s + 1) * size + at];
#pragma unroll 4
        for (uint32_t s = 0; s < a.far + (a.splits == 1); ++s) {
            const float* const from = a.far_parts + far_at(a, s, piece, key, head) + e;
            k += from[0], v += from[values];
        }
        static_cast<T*>(a.dk)[token * a.dk_token + head * a.dk_head + e] = from_f32<T>(k);
        static_cast<T*>(a.dv)[token * a.dv_token + head * a.dv_head + e] = from_f32<T>(v);
    }
}

uint32_t key_pieces(const AttentionArgs& a) { return (uint32_t)ceil_div(a.tokens, kRows) + (a.offsets ? a.sequences : 0); }

// The rows that see a tile of keys are split where there are too few tiles to fill the GPU, up
// to four workgroups for each CU: the first tiles of a text have the most rows, and with two of
// them for each CU all would wait for those.  (The gradients in us, up to two and up to
// four: 32 heads that share 8 over 8192 tokens 2977 and 2283, over 2048 264 and 246, 8192 with a
// window of 2048 1137 and 1154; eight: 1203.)  A split has 256 rows at least (1333 tokens in
// three sequences, 15 heads that share 5, a window of 300: of 128, 256, 512 rows 85, 79, 93), and
// there are 16 at most (8 heads that share one over 512 tokens: 8 splits 78, 16 68).
uint32_t splits_of(const AttentionArgs& a) {
    const uint64_t blocks = (uint64_t)key_pieces(a) * a.kv_heads;
    if (!blocks || !a.sequences) return 1;
    const uint64_t rows = std::min<uint64_t>(ceil_div(a.tokens, a.sequences), (uint64_t)a.window + kRows) * a.group;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>({1024 / blocks, rows / 256, 16}));
}

// The far rows of sinks: runs of about 1024 in a sequence of twice the average, 64 at the most,
// as far as 256 MB hold their parts and a grid its workgroups.  (32 heads that share 8 over 8192
// tokens, a window of 1024 and four sinks, in us: runs of 256 737, 512 707, 1024 719, 2048 752, one
// run 1819.)
void plan_far(AttentionGradArgs* a) {
    a->far = 0;
    if (!a->sinks || !a->sequences || a->tokens <= (uint32_t)a->window) return;
    const uint64_t listed = (uint64_t)a->sequences * a->sinks;
    a->far_packed = listed > a->tokens;
    a->far_rows = std::min<uint64_t>(listed, a->tokens);
    const uint64_t longest = std::min<uint64_t>(a->tokens, 2ull * a->tokens / a->sequences);
    const uint64_t rows = longest > (uint64_t)a->window ? (longest - a->window) * a->group : 1, bytes = std::max<uint64_t>(a->far_rows * a->kv_heads * a->dim * 8, 1);
    const uint64_t tiles = ceil_div(a->sinks, kRows) * a->sequences, pieces = key_pieces(*a);
    a->sink_tiles = tiles <= pieces ? (uint32_t)ceil_div(a->sinks, kRows) : 0;
    const uint64_t blocks = std::min(tiles, pieces) * a->kv_heads;
    a->far = (uint32_t)std::max<uint64_t>(
        1, std::min<uint64_t>({ceil_div(rows, 1024), 64, (256ull << 20) / bytes, (1ull << 22) / std::max<uint64_t>(blocks, 1)}));
}

struct Room {
    uint64_t parts, far, bytes;  // where they start
};
Room room_of(const AttentionGradArgs& a) {
    Room r;
    r.parts = ((uint64_t)a.tokens * a.heads * 12 + 15) / 16 * 16;
    r.far = r.parts + (a.splits > 1 ? ((uint64_t)a.splits * a.tokens * a.kv_heads * a.dim * 8 + 15) / 16 * 16 : 0);
    r.bytes = r.far + (a.far ? a.far + 1ull : 0) * a.far_rows * a.kv_heads * a.dim * 8;
    return r;
}

template <typename T, int D>
void launch(AttentionGradArgs a, hipStream_t stream) {
    a.pieces = (uint32_t)ceil_div((uint64_t)a.tokens * a.group, kRows) + (a.offsets ? a.sequences : 0);
    (a.vec ? attention_grad_q<T, D, true> : attention_grad_q<T, D, false>)<<<dim3(a.pieces * a.kv_heads), kWaves * 64, 0, stream>>>(a);
    if (a.far) {
        a.pieces = a.sink_tiles ? a.sink_tiles * a.sequences : key_pieces(a);
        (a.vec ? attention_grad_kv<T, D, true, true> : attention_grad_kv<T, D, false, true>)<<<dim3(a.pieces * a.kv_heads * a.far), kWaves * 64, 0, stream>>>(a);
    }
    a.pieces = key_pieces(a);
    (a.vec ? attention_grad_kv<T, D, true, false> : attention_grad_kv<T, D, false, false>)<<<dim3(a.pieces * a.kv_heads * a.splits), kWaves * 64, 0, stream>>>(a);
    if (a.splits > 1) join_kv<T><<<grid_of(ceil_div((uint64_t)a.tokens * a.kv_heads * a.dim, 256)), 256, 0, stream>>>(a);
    if (a.far) {
        a.pieces = a.sink_tiles ? a.sink_tiles * a.sequences : key_pieces(a);
        join_sinks<T><<<dim3(a.pieces * a.kv_heads), 256, 0, stream>>>(a);
    }
}

}  // namespace

uint64_t attention_grad_workspace(AttentionGradArgs a) {
    a.splits = splits_of(a);
    plan_far(&a);
    return room_of(a).bytes;
}

int32_t launch_attention_grad(AttentionGradArgs a, void* workspace, hipStream_t stream) {
    a.splits = splits_of(a);
    plan_far(&a);
    const Room room = room_of(a);
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    a.rows = reinterpret_cast<float*>(ws);
    a.parts = reinterpret_cast<float*>(ws + room.parts);
    a.far_parts = reinterpret_cast<float*>(ws + room.far);
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
