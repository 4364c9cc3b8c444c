// gfx950 kernels of attention for one new token a sequence, behind a cache.
#include <algorithm>

#include "attention.hpp"
#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"

namespace sllm {

namespace {

constexpr int kWaves = 4, kStepKeys = 32;
constexpr uint32_t kHeads = 16;           // of a workgroup
constexpr uint32_t kLeast = kWaves * 64;  // keys of a workgroup, where there are as many
constexpr uint32_t kMaxSplits = 512;

// 32 of the depth by 16 columns and 16 rows: lane (r, g) has row r and depths 8 g to 8 g + 7.
template <typename T>
__device__ __forceinline__ f32x4 multiply16(const Operand8<T>& a, const Operand8<T>& b, f32x4 acc) {
    if constexpr (__is_same(T, float)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], acc, 0, 0, 0);
        return acc;
    } else if constexpr (__is_same(T, __bf16)) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), acc, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.v), __builtin_bit_cast(f16x8, b.v), acc, 0, 0, 0);
    }
}

// The keys of a sequence: total of them, in `used` runs of `run` each, a workgroup's.
struct Split {
    int32_t total, run, used;
};
__device__ __forceinline__ Split split_keys(const AttentionArgs& a, int64_t past, uint32_t splits) {
    const int64_t window = min(past, (int64_t)a.window - 1);  // keys before the new one
    const int32_t total = (int32_t)(window + min((int64_t)a.sinks, past - window)) + 1;
    const int32_t run = (int32_t)max((total + splits - 1) / splits, kLeast);
    return {total, run, (total + run - 1) / run};
}

// Where a workgroup's part of the result goes: not divided by the sum of its weights,
// behind the largest score and that sum.
__device__ __forceinline__ uint64_t part_at(const AttentionArgs& a, uint32_t splits, uint64_t row, uint32_t split) {
    return (row * splits + split) * (a.dim + 2);
}

// Bound by reading the keys and values seen: 100003 keys of 8 heads, 410 MB, take 75 to 79 us,
// 5.2 to 5.5 TB/s, and the join 6; a copy reads and writes 5.0.  A workgroup has up to 16 heads that share
// them and a run of the keys, each of its waves a quarter of that: a wave asks for no
// other's data and waits for none.  Of 32 keys the scores are (keys x heads), the keys
// straight from memory in registers; their weights go as they come out into (elements x
// heads), the values by way of the wave's own LDS, which turns them.
template <typename T, int D, bool Vec>
__global__ __launch_bounds__(kWaves * 64) void attention_step(AttentionArgs a, uint32_t splits, float* parts) {
    typedef RowTile<T, D> Tile;
    constexpr int kSteps = D / 32, kParts = D / 16;
    constexpr uint32_t kBytes = kStepKeys * Tile::kPitch, kLoads = kStepKeys / Tile::kLoadRows;
    __shared__ __align__(16) uint8_t b0[kWaves * kBytes], b1[kWaves * kBytes];
    __shared__ float tops[kWaves][kHeads], sums[kWaves][kHeads];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 15, g = lane >> 4;
    const uint32_t head_blocks = (a.group + kHeads - 1) / kHeads;
    const uint32_t split = blockIdx.x % splits, block = blockIdx.x / splits % head_blocks, rest = blockIdx.x / splits / head_blocks;
    const uint32_t head = rest % a.kv_heads, sequence = rest / a.kv_heads;
    const uint32_t head0 = head * a.group + block * kHeads, heads = min(kHeads, a.group - block * kHeads);
    T* const out = static_cast<T*>(a.out) + (uint64_t)sequence * a.out_token;
    const int64_t past = read_length(a, sequence);
    if (past < 0) {  // takes no part
        if (splits == 1)
            for (uint32_t i = threadIdx.x; i < heads * a.dim; i += kWaves * 64) out[(head0 + i / a.dim) * a.out_head + i % a.dim] = (T)0.0f;
        return;
    }
    const Split cut = split_keys(a, past, splits);
    if ((int32_t)split >= cut.used) return;
    const KeyList keys(past, past, a.window, a.sinks);
    const int32_t first = split * cut.run, last = min(first + cut.run, cut.total);
    const int32_t slot0 = keys.lo < a.sinks ? (int32_t)(keys.lo - a.sinks) : (int32_t)((uint64_t)(keys.lo - a.sinks) % (uint32_t)a.window);
    const uint64_t cache_row = ((uint64_t)sequence * a.kv_heads + head) * a.slots;
    const T* const new_k = static_cast<const T*>(a.k) + sequence * a.k_token + head * a.k_head;
    const T* const new_v = static_cast<const T*>(a.v) + sequence * a.v_token + head * a.v_head;
    const auto row_of = [&](const void* cache, const T* fresh, int32_t i) SLLM_INLINE -> const T* {
        const int32_t k = i - keys.sinks;
        int32_t slot = k < 0 ? i : slot0 + k;
        if (k >= 0) slot = a.sinks + (slot >= a.window ? slot - a.window : slot);
        const T* p = static_cast<const T*>(cache) + (cache_row + (uint32_t)slot) * a.dim;
        return i >= last ? nullptr : i + 1 == cut.total ? fresh : p;
    };
    if (split == 0 && block == 0) {
        // the token into the slot of the one that its window leaves, which no one reads
        const uint64_t slot = past < a.sinks ? past : a.sinks + (uint64_t)(past - a.sinks) % (uint32_t)a.window;
        const uint64_t to = (cache_row + slot) * a.dim;
        for (uint32_t i = threadIdx.x; i < a.dim; i += kWaves * 64) {
            static_cast<T*>(a.cache_k)[to + i] = new_k[i];
            static_cast<T*>(a.cache_v)[to + i] = new_v[i];
        }
    }

    Operand8<T> q[kSteps];
    {
        const T* p = static_cast<const T*>(a.q) + sequence * a.q_token + (head0 + min(r, heads - 1)) * a.q_head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = load8<T, Vec>(p, 32 * s + 8 * g, a.dim);
    }
    const auto load_keys = [&](int32_t i, Operand8<T> (&k)[2][kSteps]) SLLM_INLINE {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const T* p = row_of(a.cache_k, new_k, i + 16 * n + (int32_t)r);
            if (!p) p = new_k;  // any numbers do, or none
#pragma unroll
            for (int s = 0; s < kSteps; ++s) k[n][s] = load8<T, Vec>(p, 32 * s + 8 * g, a.dim);
        }
    };
    const void* const zeros = zero_vector();
    const auto load_values = [&](int32_t i, uint8_t* to) SLLM_INLINE {
#pragma unroll
        for (uint32_t n = 0; n < kLoads; ++n) {
            const uint32_t row = n * Tile::kLoadRows + lane / Tile::kChunks, e = ((lane % Tile::kChunks) ^ Tile::turn(row)) * Tile::kElements;
            const T* p = row_of(a.cache_v, new_v, i + (int32_t)row);
            if constexpr (Vec) {
                const void* from = p + e;
                load_to_lds(p && e < a.dim ? from : zeros, to, wave * kBytes + n * 1024);
            } else {
                T v[Tile::kElements];
#pragma unroll
                for (uint32_t k = 0; k < Tile::kElements; ++k) v[k] = p && e + k < a.dim ? p[e + k] : (T)0.0f;
                lds_write(to, wave * kBytes + n * 1024 + lane * 16, __builtin_bit_cast(u32x4, v));
            }
        }
    };

    const float scale = a.scale * kLog2e;
    Reference<T> ref;
    float sum = 0;
    f32x4 acc[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) acc[d] = f32x4{0, 0, 0, 0};
    // rows 4 g + x and 16 + 4 g + x of the values, element by element
    const uint32_t columns_at =
        wave * kBytes + (sizeof(T) == 4 ? Tile::at(4 * g, r / 4) + r % 4 * 4 : Tile::at(4 * g + (lane >> 2 & 3), (lane & 3) >> 1) + (lane & 1) * 8);
    const auto values = [&](const uint8_t* from, int d) SLLM_INLINE {
        Operand8<T> o;
        const uint32_t at = opaque(columns_at ^ d * 16 * (uint32_t)sizeof(T));
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t row = 4 * g + j % 4;
                o.v[j] = lds_read<float>(from, (at ^ (Tile::turn(row) ^ Tile::turn(4 * g)) * 16) + (j / 4 * 16 + j % 4) * Tile::kPitch);
            }
        } else {
            typedef __attribute__((address_space(3))) i16x4 Lds;
            u32x2 part[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                part[u] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)((lds_u8*)from + at + u * 16 * Tile::kPitch)));
            o.v = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
        }
        return o;
    };
    const auto step = [&](int32_t i, const Operand8<T> (&k)[2][kSteps], const uint8_t* v) SLLM_INLINE {
        f32x4 s[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            s[n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < kSteps; ++e) s[n] = multiply16(k[n][e], q[e], s[n]);
        }
        if (i + kStepKeys > last)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + 16 * n + 4 * (int32_t)g + e >= last) s[n][e] = -__builtin_inff();
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e / 4][e % 4]);
        if (__any((top - ref.most) * scale > ref.kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float f = ref.raise(fmaxf(ref.most, top), scale);
            sum *= f;
#pragma unroll
            for (int d = 0; d < kParts; ++d) acc[d] *= f;
        }
        Operand8<T> p;
        const float finite = ref.finite();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w = ref.weight(s[e / 4][e % 4] - ref.less, scale, finite);
            sum += w;
            s[e / 4][e % 4] = w;
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) p.v[e] = s[e / 4][e % 4];
        } else {
            typedef T T2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                p.v[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{s[e / 2][e % 2 * 2], s[e / 2][e % 2 * 2 + 1]}, T2));
        }
#pragma unroll
        for (int d = 0; d < kParts; ++d) acc[d] = multiply16(values(v, d), p, acc[d]);
    };

    // this wave's keys, in pairs of steps
    const int32_t quarter = (cut.run + 2 * kWaves * kStepKeys - 1) / (2 * kWaves * kStepKeys) * (2 * kStepKeys);
    const int32_t i0 = first + (int32_t)wave * quarter, i1 = min(i0 + quarter, last);
    if (i0 < i1) {
        Operand8<T> ka[2][kSteps], kb[2][kSteps];
        load_keys(i0, ka);
        load_values(i0, b0);
        for (int32_t i = i0; i < i1; i += 2 * kStepKeys) {
            wait_but_loads<0>();
            wave_sync();
            if (i + kStepKeys < i1) {
                load_keys(i + kStepKeys, kb);
                load_values(i + kStepKeys, b1);
            }
            step(i, ka, b0);
            if (i + kStepKeys >= i1) break;
            wait_but_loads<0>();
            wave_sync();
            if (i + 2 * kStepKeys < i1) {
                load_keys(i + 2 * kStepKeys, ka);
                load_values(i + 2 * kStepKeys, b0);
            }
            step(i + kStepKeys, kb, b1);
        }
    }

    // The waves' parts, one after the other.
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const float exact = ref.exact(scale);
    if (g == 0) tops[wave][r] = ref.most, sums[wave][r] = sum * exact;
    __syncthreads();
    float most = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, tops[w][r]);
    const float f = ref.most == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((ref.most - most) * scale) * exact;
    static_assert(sizeof b0 >= kWaves * kHeads * 4, "");
    constexpr uint32_t kPitch = D + 4;  // floats: neighbouring heads in other banks
    float* const joined = reinterpret_cast<float*>(wave < 2 ? b0 : b1) + (wave & 1) * kHeads * kPitch;
    static_assert(sizeof b0 >= 2 * kHeads * kPitch * 4, "");
#pragma unroll
    for (int d = 0; d < kParts; ++d) *reinterpret_cast<f32x4*>(joined + r * kPitch + 16 * d + 4 * g) = acc[d] * f;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < heads * a.dim; i += kWaves * 64) {
        const uint32_t q_head = i / a.dim, e = i % a.dim;
        float top = -__builtin_inff(), total = 0, value = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w][q_head]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (tops[w][q_head] != -__builtin_inff()) total += sums[w][q_head] * __builtin_amdgcn_exp2f((tops[w][q_head] - top) * scale);
            value += reinterpret_cast<float*>(w < 2 ? b0 : b1)[((w & 1) * kHeads + q_head) * kPitch + e];
        }
        if (splits == 1) {
            out[(head0 + q_head) * a.out_head + e] = from_f32<T>(value / total);
        } else {
            float* const to = parts + part_at(a, splits, (uint64_t)sequence * a.heads + head0 + q_head, split);
            to[2 + e] = value;
            if (e == 0) to[0] = top, to[1] = total;
        }
    }
}

// The parts of a head's result: eight runs of them side by side, each in order, then those
// in order, so that every call adds in the same order (128 parts: 6.5 us, one run 65).  A lane has one element, and the
// weights of the parts are made once, by all threads.
constexpr int kRuns = 8;
template <typename T>
__global__ __launch_bounds__(128 * kRuns) void join_parts(AttentionArgs a, uint32_t splits, const float* parts) {
    __shared__ float weights[kMaxSplits], values[kRuns][128], totals[kRuns];
    const uint32_t sequence = blockIdx.x / a.heads, head = blockIdx.x % a.heads, e = threadIdx.x % 128, run = threadIdx.x / 128;
    const int64_t past = read_length(a, sequence);
    T* const out = static_cast<T*>(a.out) + sequence * a.out_token + head * a.out_head;
    if (past < 0) {
        if (threadIdx.x < a.dim) out[threadIdx.x] = (T)0.0f;
        return;
    }
    const int32_t used = split_keys(a, past, splits).used;
    const float* const from = parts + part_at(a, splits, blockIdx.x, 0);
    const uint32_t pitch = a.dim + 2;
    float top = -__builtin_inff();
    for (int32_t s = threadIdx.x; s < used; s += 128 * kRuns) weights[s] = from[s * pitch];
    __syncthreads();
    for (int32_t s = threadIdx.x % 64; s < used; s += 64) top = fmaxf(top, weights[s]);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    __syncthreads();
    for (int32_t s = threadIdx.x; s < used; s += 128 * kRuns) {
        const float at = weights[s];
        weights[s] = at == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((at - top) * (a.scale * kLog2e));
    }
    __syncthreads();
    float total = 0, value = 0;
    const int32_t end = used * (run + 1) / kRuns;
    if (e < a.dim) {
#pragma unroll 4
        for (int32_t s = used * run / kRuns; s < end; ++s) value += from[s * pitch + 2 + e] * weights[s];
        if (e == 0)
            for (int32_t s = used * run / kRuns; s < end; ++s) total += from[s * pitch + 1] * weights[s];
    }
    values[run][e] = value;
    if (e == 0) totals[run] = total;
    __syncthreads();
    if (run || e >= a.dim) return;
    value = total = 0;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) value += values[i][e], total += totals[i];
    out[e] = from_f32<T>(value / total);
}

// Workgroups that the keys of a head are split over: so many that there are two for each CU,
// if every sequence fills its cache, of 256 keys at least.  (In us, one, two and four for each
// CU: 64 sequences of 32 heads that share 8, 4096 keys each, 187, 187 and 207, one needing no
// join; one sequence of 131072 keys 101, 105 and 104; eight of up to 32768, of different
// lengths, 111, 81 and 90.)
uint32_t splits_of(const AttentionArgs& a) {
    const uint64_t alone = (uint64_t)a.sequences * a.kv_heads * ceil_div(a.group, kHeads);
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(a.slots, kLeast), kMaxSplits / alone));
}

}  // namespace

uint64_t attention_step_workspace(const AttentionArgs& a) {
    if (!a.sequences || !a.kv_heads || !a.dim) return 0;
    const uint32_t splits = splits_of(a);
    return splits > 1 ? (uint64_t)a.sequences * a.heads * splits * (a.dim + 2) * 4 : 0;
}

int32_t launch_attention_step(const AttentionArgs& a, void* workspace, hipStream_t stream) {
    const uint32_t splits = splits_of(a);
    const dim3 grid((uint32_t)(a.sequences * a.kv_heads * ceil_div(a.group, kHeads) * splits));
    float* const parts = static_cast<float*>(workspace);
    SLLM_BY_DTYPE(a.dtype, T, {
        const auto kernel = a.dim <= 64 ? (a.vec ? attention_step<T, 64, true> : attention_step<T, 64, false>)
                                        : (a.vec ? attention_step<T, 128, true> : attention_step<T, 128, false>);
        kernel<<<grid, kWaves * 64, 0, stream>>>(a, splits, parts);
        if (splits > 1) join_parts<T><<<dim3(a.sequences * a.heads), 128 * kRuns, 0, stream>>>(a, splits, parts);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
