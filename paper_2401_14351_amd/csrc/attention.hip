// gfx950 kernel of causal attention with a sliding window and sinks, over packed
// sequences or behind a cache.
#include <algorithm>

#include "attention.hpp"
#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"

namespace sllm {

namespace {

constexpr int kWaves = 4, kWaveRows = 32, kRows = kWaves * kWaveRows;

template <typename T>
constexpr int key_tile() {
    return sizeof(T) == 4 ? 32 : 64;
}

// out = softmax(scale q k^T over the keys seen) v.  One pass over the keys: a running
// maximum and sum of each row's weights, and the output rescaled where the maximum grows by
// more than 2^8.
//
// A workgroup has 128 rows of one key/value head: rows are tokens times the heads that
// share it, so that keys are read once for all of them.  A wave has 32 rows and makes the
// transposes: scores of (keys x rows), then output of (elements x rows), so that a row's
// statistics are its lane's own and weights go into the second product as they come out of
// the first.
//
// Bound by the matrix cores and the vector units in turn: of long texts (64 heads of 128
// elements that share 8, 16384 tokens, a window of 4096, bf16) 1.91 to 1.99 ms in a row, 0.97 to
// 1.0 PF/s (each from an idle GPU 2.04 to 2.17), where the library's large products reach 1.4;
// the matrix cores are busy 47 % of the cycles, the vector units 42 %, LDS 24 % without
// conflicts.  In 32 bits 85 TF/s of 154 (packed texts, as below).  Two workgroups a CU, since a
// wave takes 240 registers, hide each other's loads; tiles of 64 keys keep the registers so
// (32 in 32 bits).  Making the scores of the next 32 keys beside the weights of these was
// slower (2253 us to 2012, and 8191 tokens in 32 heads, a window of 1024, 234 to 187): the
// compiler needs the registers.  8191 tokens in five sequences take 162 us, 0.59 PF/s: 69
// pieces of 32 heads for 512 places, 4.3 rounds, the last a third full, of which each piece
// starts and ends alone.
template <typename T, int D, bool Vec, bool Cached>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) * D > 256 ? 1 : 2) void attention_rows(AttentionArgs a) {
    constexpr int kKeys = key_tile<T>(), kSteps = D / 16, kParts = D / 32;
    constexpr uint32_t kBytes = kKeys * RowTile<T, D>::kPitch;
    __shared__ __align__(16) uint8_t k0[kBytes], v0[kBytes], k1[kBytes], v1[kBytes];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = lane & 31, h = lane >> 5;

    const uint32_t index = xcd_index();
    const uint32_t head = index / a.pieces;  // of keys and values
    const Piece piece = find_piece(a.offsets, a.wide_offsets, a.sequences, a.tokens, a.group, kRows, index % a.pieces, a.pieces);
    T* const out = static_cast<T*>(a.out);
    int64_t past = 0;
    if (Cached && piece.n) past = read_length(a, piece.sequence);
    if (!piece.n || past < 0) {
        // tokens of no sequence, or of one that takes no part
        Piece none = piece;
        uint32_t tokens = a.tokens;
        if (piece.n) none.spare = (uint32_t)(((uint64_t)piece.n * a.group + kRows - 1) / kRows), tokens = none.n;
        T* const from = out + (piece.n ? piece.first * a.out_token : 0);
        if (piece.n) none.first = none.past_end = 0;
        clear_spare(none, tokens, from, a.out_token, a.out_head, head * a.group, a.group, a.dim);
        if (!Cached && a.lse) clear_spare(none, tokens, a.lse, a.heads, 1, head * a.group, a.group, 1);
        return;
    }
    const uint32_t rows = piece.n * a.group;  // fewer than 2^32
    // the last pieces see the most keys: they come first
    const uint32_t row0 = ((rows - 1) / kRows - piece.piece) * kRows, row1 = min(row0 + kRows, rows) - 1;
    const uint32_t t0 = row0 / a.group, t1 = row1 / a.group;
    const KeyList keys(past + t0, past + t1, a.window, a.sinks);
    const int32_t base = (int32_t)(past + t0 - keys.lo) - (int32_t)t0;  // a token's position from lo on, less the token

    // this wave's rows, the last one again past the end
    const uint32_t wave_row = row0 + wave * kWaveRows, row = min(wave_row + c, rows - 1);
    const uint32_t token = row / a.group, q_head = head * a.group + row % a.group;
    const KeyList::Sight sight = keys.sight(base + (int32_t)token);
    const int32_t at0 = base + (int32_t)(min(wave_row, rows - 1) / a.group), at1 = base + (int32_t)(min(wave_row + 31, rows - 1) / a.group);
    Operand8<T> q[kSteps];
    {
        const T* p = static_cast<const T*>(a.q) + (uint64_t)(piece.first + token) * a.q_token + q_head * a.q_head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = load8<T, Vec>(p, 16 * s + 8 * h, a.dim);
    }

    // where key i's row is
    const int32_t held = Cached ? (int32_t)(past - keys.lo) : 0;  // keys from lo on in the cache
    const int32_t past_sinks = Cached ? (int32_t)min(past, (int64_t)1 << 30) : 0;
    int32_t slot0 = 0;                                             // the slot of lo, among the window's
    if (Cached) slot0 = keys.lo < a.sinks ? (int32_t)(keys.lo - a.sinks) : (int32_t)((uint64_t)(keys.lo - a.sinks) % (uint32_t)a.window);
    const uint64_t cache_row = Cached ? ((uint64_t)piece.sequence * a.kv_heads + head) * a.slots : 0;
    const auto key_row = [&](const void* fresh, uint64_t token_stride, uint64_t head_stride, const void* cache, int32_t i) SLLM_INLINE -> const T* {
        const bool none = i >= keys.total;
        i = min(i, keys.total - 1);
        const int32_t k = i - keys.sinks;
        const T* const rows_of = static_cast<const T*>(fresh) + head * head_stride;
        if constexpr (!Cached) {
            const uint32_t token = k < 0 ? (uint32_t)i : (uint32_t)((int32_t)keys.lo + k);
            const T* p = rows_of + (uint64_t)(piece.first + token) * token_stride;
            return none ? nullptr : p;
        } else {
            const int32_t fresh_one = k < 0 ? i - past_sinks : k - held;  // of this call's tokens, or before them
            const T* p = rows_of + (uint64_t)(piece.first + (uint32_t)max(fresh_one, 0)) * token_stride;
            int32_t slot = k < 0 ? i : slot0 + k;
            if (k >= 0) slot = a.sinks + (slot >= a.window ? slot - a.window : slot);
            p = fresh_one >= 0 ? p : static_cast<const T*>(cache) + (cache_row + (uint32_t)slot) * a.dim;
            return none ? nullptr : p;
        }
    };
    // Tiles whose keys lie one behind the other need no look at each.
    const bool repeats = Vec && a.dim == D && (Cached || max(a.k_token, a.v_token) < (1u << 24));
    LaneOffsets<T, D, kKeys, kWaves> k_at, v_at;
    if constexpr (Vec) {
        const uint32_t k_token = Cached ? D : (uint32_t)a.k_token, v_token = Cached ? D : (uint32_t)a.v_token;
        k_at.set(k_at.kRun * (uint64_t)k_token, [&](uint32_t r) SLLM_INLINE { return r * k_token; });
        v_at.set(v_at.kRun * (uint64_t)v_token, [&](uint32_t r) SLLM_INLINE { return r * v_token; });
    }
    const auto stage = [&](int32_t i0, uint8_t* k, uint8_t* v) SLLM_INLINE {
        if constexpr (Cached) {
            // in the window and in the cache, all before its end or all behind it
            const int32_t n = i0 - keys.sinks, at = slot0 + n;
            if (repeats && n >= 0 && n + kKeys <= held && (at >= a.window || at + kKeys <= a.window)) {
                const uint64_t row = cache_row + (uint32_t)(a.sinks + (at >= a.window ? at - a.window : at));
                k_at.stage(k, static_cast<const T*>(a.cache_k) + row * D);
                v_at.stage(v, static_cast<const T*>(a.cache_v) + row * D);
                return;
            }
        } else if (repeats && i0 >= keys.sinks && i0 + kKeys <= keys.total) {
            const uint64_t token = piece.first + (uint32_t)((int32_t)keys.lo + i0 - keys.sinks);
            k_at.stage(k, static_cast<const T*>(a.k) + head * a.k_head + token * a.k_token);
            v_at.stage(v, static_cast<const T*>(a.v) + head * a.v_head + token * a.v_token);
            return;
        }
        stage_rows<T, D, kKeys, kWaves, Vec>(k, a.dim, [&](uint32_t r) SLLM_INLINE { return key_row(a.k, a.k_token, a.k_head, a.cache_k, i0 + (int32_t)r); });
        stage_rows<T, D, kKeys, kWaves, Vec>(v, a.dim, [&](uint32_t r) SLLM_INLINE { return key_row(a.v, a.v_token, a.v_head, a.cache_v, i0 + (int32_t)r); });
    };

    const float scale = a.scale * kLog2e;
    Reference<T> ref;
    bool far = false;  // a row's scores are too large to be scaled as they are
    float sum = 0;
    f32x16 acc[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) acc[d] = f32x16{};
    const uint32_t rows_at = rows_from<T, D>(lane), columns_at = columns_from<T, D>(lane);

    bool out_of_sight = false;  // something was taken out
    const auto tile = [&](int32_t i0, const uint8_t* k, const uint8_t* v, bool masked) SLLM_INLINE {
        bool bad = false;
        f32x16 s[kKeys / 32];
        RowFragments<T, D> kf[kKeys / 32];
        ColumnFragments<T, D, kKeys> vf;
        kf[0].read(k, rows_at, 0);
        phase();
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int n = 0; n < kKeys / 32; ++n) {
            if (n + 1 < kKeys / 32)
                kf[n + 1].read(k, rows_at, 32 * (n + 1));
            else
                vf.read(v, columns_at, 0, 0);
            s[n] = kf[n].times(q);
            phase();
        }
        __builtin_amdgcn_s_setprio(0);
        if (masked) {
            const KeyList::Sight here = sight.here();
#pragma unroll
            for (int n = 0; n < kKeys / 32; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[n][i] = here.sees(i0 + 32 * n + 8 * (i / 4) + 4 * (int32_t)h + i % 4) ? s[n][i] : -__builtin_inff();
            bad = any_not_finite<T, D, kKeys>(v);
            out_of_sight |= bad;
        }
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < kKeys / 32; ++n)
#pragma unroll
            for (int i = n == 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
        if (__any((top - ref.most) * scale > ref.kSlack)) {
            const f32x2 tops = both_halves(top);
            const float f = ref.raise(fmaxf(ref.most, fmaxf(tops[0], tops[1])), scale);
            far = __any(ref.less != 0);
            sum *= f;
#pragma unroll
            for (int d = 0; d < kParts; ++d) acc[d] *= f;
        }
        if (far)
#pragma unroll
            for (int n = 0; n < kKeys / 32; ++n) s[n] -= ref.less;
        Operand8<T> p[kKeys / 16];
        const float finite = ref.finite();
        float part = 0;
#pragma unroll
        for (int n = 0; n < kKeys / 32; ++n) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[n][i] = ref.weight(s[n][i], scale, finite);
                part += s[n][i];
            }
            p[2 * n] = as_operand<T>(s[n], 0);
            p[2 * n + 1] = as_operand<T>(s[n], 1);
        }
        sum += part;
        phase();
        __builtin_amdgcn_s_setprio(1);
        add_weighted<T, D, kKeys>(acc, vf, v, columns_at, 0, p, bad);
        __builtin_amdgcn_s_setprio(0);
    };
    const auto step = [&](int32_t i0, const uint8_t* k, const uint8_t* v, uint8_t* next_k, uint8_t* next_v) SLLM_INLINE {
        wait_but_loads<0>();
        barrier();  // this tile has landed, and all waves are done with the other one
        if (i0 + kKeys < keys.total) stage(i0 + kKeys, next_k, next_v);
        if (!keys.none(at0, at1, i0, i0 + kKeys - 1)) tile(i0, k, v, !keys.all(at0, at1, i0, i0 + kKeys - 1));
    };
    stage(0, k0, v0);
    for (int32_t i0 = 0; i0 < keys.total; i0 += 2 * kKeys) {
        step(i0, k0, v0, k1, v1);
        if (i0 + kKeys < keys.total) step(i0 + kKeys, k1, v1, k0, v0);
    }

    if (out_of_sight)
        for (int32_t i = 0; i < keys.total; ++i)
            put_back<T, D>(acc, key_row(a.v, a.v_token, a.v_head, a.cache_v, i), a.dim, sight.sees(i));
    const f32x2 sums = both_halves(sum);
    sum = sums[0] + sums[1];
    if (wave_row + c >= rows) return;
    const uint64_t out_row = piece.first + token;
    if (a.lse && h == 0) a.lse[out_row * a.heads + q_head] = ref.log_sum(sum, scale) * kLn2;
    store_column<T, D, Vec>(acc, 1.0f / sum, out + out_row * a.out_token + q_head * a.out_head, a.dim);
}

// The new tokens of each sequence into its cache, after the attention that still reads
// what they replace: of those that share a slot the last one alone.  Bound by the reads that
// follow one another, of offsets and then rows: 1200 tokens of 8 heads, 10 MB, 6.2 us.
template <typename W>
__global__ __launch_bounds__(256) void write_cache(AttentionArgs a, uint32_t row_words) {
    // the tokens of sequence blockIdx.x; what is read is asked for at once
    __shared__ uint32_t bounds[4];
    const auto clamp = [&](int64_t v) { return (uint32_t)min(max(v, (int64_t)0), (int64_t)a.tokens); };
    const uint32_t s = blockIdx.x;
    const int64_t past = read_length(a, s);
    const uint32_t end = clamp(read_id(a.offsets, a.wide_offsets, s + 1));
    uint32_t most = 0;
    for (uint32_t i = threadIdx.x; i <= s; i += 256) most = max(most, clamp(read_id(a.offsets, a.wide_offsets, i)));
#pragma unroll
    for (uint32_t lanes = 32; lanes; lanes /= 2) most = max(most, (uint32_t)__shfl_xor((int)most, lanes));
    if (threadIdx.x % 64 == 0) bounds[threadIdx.x / 64] = most;
    __syncthreads();
    const uint32_t first = max(max(bounds[0], bounds[1]), max(bounds[2], bounds[3])), n = max(first, end) - first;
    if (past < 0) return;
    const uint32_t size = sizeof(W) / a.element;  // strides are in elements
    for (uint32_t t = blockIdx.y; t < n; t += gridDim.y) {
        const int64_t p = past + t;
        if (p >= a.sinks && p + a.window < past + n) continue;  // a later one has its slot
        const uint64_t slot = p < a.sinks ? p : a.sinks + (uint64_t)(p - a.sinks) % (uint32_t)a.window;
        const uint64_t to = ((uint64_t)s * a.kv_heads * a.slots + slot) * row_words;
        const W* const k = static_cast<const W*>(a.k) + (uint64_t)(first + t) * a.k_token / size;
        const W* const v = static_cast<const W*>(a.v) + (uint64_t)(first + t) * a.v_token / size;
        for (uint32_t i = threadIdx.x; i < a.kv_heads * row_words; i += 256) {
            const uint32_t head = i / row_words, w = i - head * row_words;
            const uint64_t at = to + (uint64_t)head * a.slots * row_words + w;
            const W key = k[head * a.k_head / size + w], value = v[head * a.v_head / size + w];
            static_cast<W*>(a.cache_k)[at] = key;
            static_cast<W*>(a.cache_v)[at] = value;
        }
    }
}

template <typename T, int D>
void launch(const AttentionArgs& a, bool vec, dim3 grid, hipStream_t stream) {
    const auto kernel = a.cache_k ? (vec ? attention_rows<T, D, true, true> : attention_rows<T, D, false, true>)
                                  : (vec ? attention_rows<T, D, true, false> : attention_rows<T, D, false, false>);
    kernel<<<grid, kWaves * 64, 0, stream>>>(a);
}

}  // namespace

int32_t launch_attention(AttentionArgs a, hipStream_t stream) {
    a.pieces = (uint32_t)(ceil_div((uint64_t)a.tokens * a.group, kRows) + (a.offsets ? a.sequences : 0));
    const dim3 grid(a.pieces * a.kv_heads);
    SLLM_BY_DTYPE(a.dtype, T, {
        if (a.dim <= 64)
            launch<T, 64>(a, a.vec, grid, stream);
        else
            launch<T, 128>(a, a.vec, grid, stream);
    });
    SLLM_HIP(hipGetLastError());
    if (a.cache_k && a.sequences) {
        a.element = a.dtype == SLLM_DTYPE_F32 ? 4 : 2;
        const uint32_t row_bytes = a.dim * a.element;
        // a workgroup for each of its tokens, were one sequence to have a few hundred (one for
        // 4096 vectors of them, of 8 sequences with 1200 in all, takes 10.5 us instead of 6.2)
        const dim3 blocks(a.sequences, std::min<uint32_t>(a.tokens, a.sequences > 64 ? 16 : 256));
        if (a.vec)
            write_cache<u32x4><<<blocks, 256, 0, stream>>>(a, row_bytes / 16);
        else if (a.element == 4)
            write_cache<uint32_t><<<blocks, 256, 0, stream>>>(a, row_bytes / 4);
        else
            write_cache<uint16_t><<<blocks, 256, 0, stream>>>(a, row_bytes / 2);
        SLLM_HIP(hipGetLastError());
    }
    return SLLM_OK;
}

}  // namespace sllm
