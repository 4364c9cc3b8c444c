// gfx950 kernels of token embeddings: the lookup of table rows (and the
// dequantisation of a whole matrix, a lookup of every row in turn) and its
// gradient.
#include <algorithm>
#include <utility>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

namespace {

struct Ids {
    const void* p;
    bool wide;
};

// Id i, or -1 where it names none of `vocab` rows.
__device__ __forceinline__ int32_t id_at(const Ids& ids, uint64_t i, uint32_t vocab) {
    const int64_t v = ids.wide ? static_cast<const int64_t*>(ids.p)[i] : static_cast<const int32_t*>(ids.p)[i];
    return v < 0 || v >= (int64_t)vocab ? -1 : (int32_t)v;
}

struct Lookup {
    Operand table;
    uint32_t vocab, dim;
    Ids ids;
    uint64_t n;
    float scale;
    uint64_t out_stride;
    uint32_t lanes;  // of a row: 32, 64 or 256
};

// Columns c .. c + 7 of a row, those past the end zero.  Vec: rows start on 16
// bytes and end on a multiple of eight columns.
template <bool Vec, typename S>
__device__ __forceinline__ void load8(const S* row, uint32_t c, uint32_t dim, float (&v)[8]) {
    S e[8];
    if constexpr (Vec) {
        u32x4 raw[sizeof(S) / 2];
#pragma unroll
        for (uint32_t i = 0; i < sizeof(S) / 2; ++i) raw[i] = reinterpret_cast<const u32x4*>(row + c)[i];
        __builtin_memcpy(e, raw, sizeof e);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) e[i] = c + i < dim ? row[c + i] : (S)0.0f;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = to_f32(e[i]);
}

template <bool Vec, typename T>
__device__ __forceinline__ void store8(T* row, uint32_t c, uint32_t dim, const float (&v)[8]) {
    T e[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) e[i] = from_f32<T>(v[i]);
    if constexpr (Vec) {
        u32x4 raw[sizeof(T) / 2];
        __builtin_memcpy(raw, e, sizeof e);
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<u32x4*>(row + c)[i] = raw[i];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (c + i < dim) row[c + i] = e[i];
    }
}

// out[i] = scale table[ids[i]], the product in 32 bits.  Eight columns a lane,
// `lanes` of them a row at a time: 16 bytes a store, and of a row in MX FP4 a word
// of codes.  Bound by memory: 8191 rows of 8192 columns from bfloat16 54 us, 5.0
// TB/s, from MX FP4 36 us, 4.7 TB/s (25 where the last-level cache has the table);
// 16 rows are bound by their two loads one after the other, 3 us.  S: the table's
// elements, void for MX FP4.  Vec: rows start on 16 bytes and end on a multiple of eight
// columns.
template <bool Vec, typename S, typename T>
__global__ __launch_bounds__(256) void lookup(Lookup a, T* out) {
    const uint64_t i = (uint64_t)block_index() * (256 / a.lanes) + threadIdx.x / a.lanes;
    if (i >= a.n) return;
    const int64_t row = a.ids.p ? id_at(a.ids, i, a.vocab) : (int64_t)i;
    const uint32_t blocks = (a.dim + 31) / 32, pitch = (blocks + 15) / 16 * 16;
    // A word of codes a lane does not fill the memory's latency: several are under way
    // (8191 rows of 8192 from cold memory 36 us, one at a time 43; rows of 2048, where a
    // lane has one word, 27.7 and 26.4).
    constexpr uint32_t kTogether = __is_same(S, void) ? 4 : 1;
    for (uint32_t c0 = threadIdx.x % a.lanes * 8; c0 < a.dim; c0 += kTogether * a.lanes * 8) {
        float v[kTogether][8] = {};
        if (row >= 0) {
            if constexpr (__is_same(S, void)) {
                uint32_t codes[kTogether] = {}, scales[kTogether] = {};
#pragma unroll
                for (uint32_t u = 0; u < kTogether; ++u) {
                    if (u * a.lanes * 8 >= a.dim) break;  // short rows have none of these
                    const uint32_t c = min(c0 + u * a.lanes * 8, a.dim - 1) & ~7u;
                    codes[u] = *reinterpret_cast<const uint32_t*>(a.table.codes + (uint64_t)row * blocks * 16 + c / 2);
                    scales[u] = a.table.scales[(uint64_t)row * pitch + c / 32];
                }
#pragma unroll
                for (uint32_t u = 0; u < kTogether; ++u) {
                    const float scale = mx_scale(scales[u]);
                    const f32x2 two[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], scale, 0),
                                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], scale, 1),
                                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], scale, 2),
                                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], scale, 3)};
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) v[u][e] = two[e / 2][e % 2];
                }
            } else {
#pragma unroll
                for (uint32_t u = 0; u < kTogether; ++u)
                    load8<Vec>(static_cast<const S*>(a.table.data) + (uint64_t)row * a.table.stride, c0, a.dim, v[u]);
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kTogether; ++u) {
            const uint32_t c = c0 + u * a.lanes * 8;
            if (c >= a.dim) break;
            if (row >= 0)  // else zeros, whatever the scale
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) v[u][e] *= a.scale;
            store8<Vec>(out + i * a.out_stride, c, a.dim, v[u]);
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient: positions sorted by token, then sums over runs of equal tokens
// ---------------------------------------------------------------------------

// A key is a token and its position; ids that name no row sort last, as token
// `vocab`.  Keys differ, so their order is one and the same however it is found.
constexpr uint32_t kSortTile = 1024;  // keys a workgroup sorts
constexpr uint32_t kMergeRuns = 16;   // sorted runs merged at once, a lane each
// Sorted positions that the same lanes sum.  Twice as many leave half the sums to
// join but take longer themselves: 16,384 positions are the same to 2 us either way.
constexpr uint32_t kWindow = 16;
constexpr uint32_t kZeroRows = 16;    // table rows a workgroup looks up and clears, 16 lanes each

__device__ __forceinline__ uint32_t token_of(uint64_t key) { return (uint32_t)(key >> 32); }

// x of the lane that differs in bit J (1 to 32) of its number.
template <int J>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
    if constexpr (J == 1) return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xF, 0xF, true);       // quads in the order 1 0 3 2
    if constexpr (J == 2) return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xF, 0xF, true);       // 2 3 0 1
    if constexpr (J == 8) return __builtin_amdgcn_mov_dpp(x, 0x128, 0xF, 0xF, true);      // rows of 16 turned by 8
    if constexpr (J == 4 || J == 16) return __builtin_amdgcn_ds_swizzle(x, 0x1F | J << 10);  // within 32 lanes
    if constexpr (J == 32) return __shfl_xor(x, 32);
}

// One step of a bitonic sort: the lower of two keys J apart goes to the lane
// without bit J where K's bit is clear.
template <uint32_t K, uint32_t J>
__device__ __forceinline__ void sort_step(uint32_t t, uint32_t& key, uint32_t* keys) {
    uint32_t other;
    if constexpr (J >= 64) {
        __syncthreads();
        keys[t] = key;
        __syncthreads();
        other = keys[t ^ J];
    } else {
        other = lane_xor<J>(key);
    }
    const bool lower = ((t & J) == 0) == ((t & K) == 0);
    key = lower ? min(key, other) : max(key, other);
    if constexpr (J > 1) sort_step<K, J / 2>(t, key, keys);
}

template <uint32_t K = 2>
__device__ __forceinline__ void sort_tile(uint32_t t, uint32_t& key, uint32_t* keys) {
    sort_step<K, K / 2>(t, key, keys);
    if constexpr (K < kSortTile) sort_tile<2 * K>(t, key, keys);
}

// Bitonic sort of a tile, a key a lane: partners up to 32 lanes away by lane
// exchanges, the others through LDS.  A tile's key is the token and ten bits of
// the position in 32 bits, where the table has fewer than 2^22 rows; 2,048 ids
// then take 5.1 us, 9.4 with keys of 64 bits.
__global__ __launch_bounds__(1024) void sort_tiles(Ids ids, uint32_t n, uint32_t vocab, uint64_t* out) {
    __shared__ uint32_t keys[kSortTile];
    const uint32_t t = threadIdx.x, first = blockIdx.x * kSortTile, i = first + t;
    uint32_t key = ~0u;  // past the ids: after all of them
    if (i < n) {
        const int32_t id = id_at(ids, i, vocab);
        key = (id < 0 ? vocab : (uint32_t)id) << 10 | t;
    }
    sort_tile(t, key, keys);
    if (i < n) out[i] = (uint64_t)(key >> 10) << 32 | (first + (key & 1023));
}

__global__ __launch_bounds__(1024) void sort_tiles_wide(Ids ids, uint32_t n, uint32_t vocab, uint64_t* out) {
    __shared__ uint64_t keys[kSortTile];
    const uint32_t t = threadIdx.x, i = blockIdx.x * kSortTile + t;
    uint64_t key = ~0ull;
    if (i < n) {
        const int32_t id = id_at(ids, i, vocab);
        key = (uint64_t)(id < 0 ? vocab : (uint32_t)id) << 32 | i;
    }
    for (uint32_t k = 2; k <= kSortTile; k *= 2)
        for (uint32_t j = k / 2; j > 0; j /= 2) {
            __syncthreads();
            keys[t] = key;
            __syncthreads();
            const uint64_t other = keys[t ^ j];
            const bool lower = ((t & j) == 0) == ((t & k) == 0);
            key = lower == (key < other) ? key : other;
        }
    if (i < n) out[i] = key;
}

// Merge groups of kMergeRuns sorted runs: a key's place is the number of
// smaller keys in its group, found by one bisection per run, a lane each.  Bound
// by the bisections' loads from L2: 16,384 keys 6.5 us (with three probes at a time
// instead of one there are fewer loads in a row but more in all, and it is 8 us).
__global__ __launch_bounds__(256) void merge_runs(const uint64_t* in, uint32_t n, uint32_t run, uint64_t* out) {
    const uint64_t i = ((uint64_t)blockIdx.x * 256 + threadIdx.x) / kMergeRuns;
    const uint32_t q = threadIdx.x % kMergeRuns;
    if (i >= n) return;
    const uint64_t key = in[i];
    const uint64_t group = i / run / kMergeRuns * kMergeRuns * run;
    const uint64_t first = group + (uint64_t)q * run;
    uint32_t count = 0;
    if (first < n) {
        uint64_t lo = first, hi = min(first + run, (uint64_t)n);
        while (lo < hi) {
            const uint64_t mid = (lo + hi) / 2;
            if (in[mid] < key)
                lo = mid + 1;
            else
                hi = mid;
        }
        count = (uint32_t)(lo - first);
    }
    for (uint32_t d = kMergeRuns / 2; d > 0; d /= 2) count += __shfl_xor(count, d);
    if (q == 0) out[group + count] = key;
}

struct GradArgs {
    const uint64_t* keys;  // sorted
    uint32_t n, vocab, dim;
    float scale;
    uint64_t dy_stride, grad_stride;
    bool accumulate;
    float* partial;        // a window's first and last run: [windows][2][pitch]
    uint32_t pitch, windows;
    uint32_t lanes;        // of a row: 32, 64 or 256
    uint32_t chunks;       // of a row, lanes * 8 columns each
    uint32_t sum_blocks;   // workgroups that sum; the rest clear rows
    // of a row to clear: its bytes, those a lane stores at once (16, 4 or 2), and its lanes (a power of two)
    uint64_t row_bytes;
    uint32_t unit, clear_lanes;
};

template <typename U>
__device__ __forceinline__ void clear_row(uint8_t* row, uint64_t bytes, uint32_t lane, uint32_t lanes) {
    for (uint64_t i = lane; i < bytes / sizeof(U); i += lanes) reinterpret_cast<U*>(row)[i] = U{};
}

// A table row's gradient from its whole sum.
template <bool Vec, typename T>
__device__ __forceinline__ void write_row(const GradArgs& a, T* grad, uint32_t token, uint32_t c, float (&sum)[8]) {
    T* row = grad + (uint64_t)token * a.grad_stride;
    float old[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (a.accumulate) load8<Vec>(row, c, a.dim, old);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) sum[i] = old[i] + sum[i] * a.scale;
    store8<Vec>(row, c, a.dim, sum);
}

// grad[v] = scale times the sum of dy over the positions of v, in 32 bits.  Sorting
// the positions first makes the order of a sum, and so its bits, the same on every
// run, which atomic sums are not, and no row is read or written twice.
//
// Bound by memory: 16,384 rows of 4096 in bfloat16 into 32,000 (134 MB in, 262 MB
// out) 79 us, 5.0 TB/s.
//
// The first workgroups take windows of sorted positions.  A run of equal tokens
// inside one window becomes its row at once; one that goes on into the next
// window, or came from the one before, leaves its sum for join_runs.  The other
// workgroups clear the rows that no key names, each row looked for by 16 lanes:
// the search is a chain of loads that nothing can be written before the end of.
template <bool Vec, typename S, typename T>
__global__ __launch_bounds__(256) void sum_runs(GradArgs a, const S* dy, T* grad) {
    const uint32_t block = block_index();
    if (block >= a.sum_blocks) {
        __shared__ uint32_t named[kZeroRows];
        const uint32_t row0 = (block - a.sum_blocks) * kZeroRows;
        if (a.accumulate || row0 >= a.vocab) return;  // of the workgroups launched beyond those asked for
        const uint32_t probe = threadIdx.x % 16, token = row0 + threadIdx.x / 16;
        const uint64_t key = (uint64_t)token << 32;
        uint32_t lo = 0, hi = a.n;  // the first key of the token or a later one is in [lo, hi]
        while (__any(lo < hi)) {
            const uint32_t step = (hi - lo) / 17 + 1;
            const uint64_t at = lo + (uint64_t)(probe + 1) * step - 1;
            const uint64_t less = __ballot(at < hi && a.keys[at] < key);
            const uint32_t count = __popc((uint32_t)(less >> (threadIdx.x & 48)) & 0xffff);
            hi = (uint32_t)min((uint64_t)hi, lo + (uint64_t)(count + 1) * step - 1);
            lo += count * step;
        }
        if (probe == 0) named[threadIdx.x / 16] = lo < a.n && token_of(a.keys[lo]) == token;
        __syncthreads();
        const uint32_t lane = threadIdx.x & (a.clear_lanes - 1), shift = __builtin_ctz(a.clear_lanes);
        for (uint32_t r = threadIdx.x >> shift; r < kZeroRows && row0 + r < a.vocab; r += 256u >> shift) {
            if (named[r]) continue;
            uint8_t* row = reinterpret_cast<uint8_t*>(grad + (uint64_t)(row0 + r) * a.grad_stride);
            if (a.unit == 16)
                clear_row<u32x4>(row, a.row_bytes, lane, a.clear_lanes);
            else if (a.unit == 4)
                clear_row<uint32_t>(row, a.row_bytes, lane, a.clear_lanes);
            else
                clear_row<uint16_t>(row, a.row_bytes, lane, a.clear_lanes);
        }
        return;
    }
    const uint32_t per = 256 / a.lanes;  // windows of a workgroup
    const uint32_t w = block / a.chunks * per + threadIdx.x / a.lanes;
    const uint32_t c = (block % a.chunks * a.lanes + threadIdx.x % a.lanes) * 8;
    if (w >= a.windows || c >= a.dim) return;
    const uint32_t first = w * kWindow, end = min(first + kWindow, a.n);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    uint32_t token = token_of(a.keys[first]);
    bool whole = first == 0 || token_of(a.keys[first - 1]) != token;  // the run starts here
    // rows are loaded some ahead of the sum, which a change of token holds up
    constexpr uint32_t kAhead = 4;
    for (uint32_t i0 = first; i0 < end; i0 += kAhead) {
        uint64_t keys[kAhead];
        float v[kAhead][8];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
            keys[u] = a.keys[min(i0 + u, end - 1)];
            const uint64_t position = token_of(keys[u]) < a.vocab ? (uint32_t)keys[u] : 0;
            load8<Vec>(dy + position * a.dy_stride, c, a.dim, v[u]);
        }
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
            if (i0 + u >= end) break;
            if (token_of(keys[u]) != token) {
                if (whole)
                    write_row<Vec>(a, grad, token, c, sum);
                else
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) a.partial[(uint64_t)w * 2 * a.pitch + c + e] = sum[e];
                token = token_of(keys[u]);
                whole = true;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) sum[e] = 0;
            }
            if (token >= a.vocab) return;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) sum[e] += v[u][e];
        }
    }
    const bool goes_on = end < a.n && token_of(a.keys[end]) == token;
    if (whole && !goes_on)
        write_row<Vec>(a, grad, token, c, sum);
    else
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) a.partial[((uint64_t)w * 2 + whole) * a.pitch + c + e] = sum[e];
}

// The rows of runs that cross windows: the last run of the window where it
// starts, then the first of each window it goes on into.  Bound by the longest
// run: of 16,384 positions of text one token in ten is the same, 12 us.
template <bool Vec, typename T>
__global__ __launch_bounds__(256) void join_runs(GradArgs a, T* grad) {
    const uint32_t per = 256 / a.lanes;
    const uint32_t w = blockIdx.x / a.chunks * per + threadIdx.x / a.lanes;
    const uint32_t c = (blockIdx.x % a.chunks * a.lanes + threadIdx.x % a.lanes) * 8;
    if (w + 1 >= a.windows) return;
    const uint32_t first = w * kWindow, end = first + kWindow;
    const uint32_t token = token_of(a.keys[end - 1]);
    if (token >= a.vocab || token_of(a.keys[end]) != token) return;            // ends here
    if (token_of(a.keys[first]) == token && first && token_of(a.keys[first - 1]) == token) return;  // starts before
    // how many windows it goes on into, 32 looked at together (a row has that many lanes or more)
    const uint32_t lane = threadIdx.x % 64, half = lane & 32;
    uint32_t last = w;
    for (uint32_t found = 32; found == 32; last += found) {
        const uint64_t next = last + 1 + (uint64_t)(lane & 31);
        const uint64_t same = __ballot(next < a.windows && token_of(a.keys[next * kWindow]) == token);
        const uint32_t mine = (uint32_t)(same >> half);
        found = ~mine ? __builtin_ctz(~mine) : 32;
    }
    if (c >= a.dim) return;
    const float* p = a.partial + ((uint64_t)w * 2 + 1) * a.pitch + c;
    f32x4 lo = reinterpret_cast<const f32x4*>(p)[0], hi = reinterpret_cast<const f32x4*>(p)[1];
    p += a.pitch;
    uint32_t next = w + 1;
    // a frequent token's run is a hundred windows long, and each is a load from far away
    constexpr uint32_t kTogether = 16;
    for (; next + kTogether <= last + 1; next += kTogether) {
        f32x4 far[kTogether][2];
#pragma unroll
        for (uint32_t i = 0; i < kTogether; ++i, p += 2 * (uint64_t)a.pitch)
#pragma unroll
            for (int e = 0; e < 2; ++e) far[i][e] = reinterpret_cast<const f32x4*>(p)[e];
#pragma unroll
        for (uint32_t i = 0; i < kTogether; ++i) {
            lo += far[i][0];
            hi += far[i][1];
        }
    }
#pragma unroll 8
    for (; next <= last; ++next, p += 2 * (uint64_t)a.pitch) {
        lo += reinterpret_cast<const f32x4*>(p)[0];
        hi += reinterpret_cast<const f32x4*>(p)[1];
    }
    float sum[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    write_row<Vec>(a, grad, token, c, sum);
}

}  // namespace

namespace {

uint64_t element_bytes(uint32_t dtype) { return dtype == SLLM_DTYPE_F32 ? 4 : 2; }

// Rows at this address, apart by this stride, start on 16 bytes.
bool on_vectors(const void* data, uint64_t rows, uint64_t stride, uint32_t dtype) {
    return reinterpret_cast<uintptr_t>(data) % 16 == 0 && (rows <= 1 || stride * element_bytes(dtype) % 16 == 0);
}

// Lanes that take a row together, eight columns each: a workgroup for long rows
// (512 rows of 4096 looked up in 3.6 us, by a wave each 4.7), a wave or half of one
// for others (16384 of 768 9.8, by workgroups 12.4; of 256 4.6, by waves 5.4).
uint32_t row_lanes(uint64_t dim) { return dim > 1024 ? 256 : dim > 256 ? 64 : 32; }

template <bool Vec, typename T>
void launch_lookup(const Lookup& l, dim3 grid, T* out, hipStream_t stream) {
    if (l.table.codes)
        lookup<Vec, void, T><<<grid, 256, 0, stream>>>(l, out);
    else
        SLLM_BY_DTYPE(l.table.dtype, S, (lookup<Vec, S, T><<<grid, 256, 0, stream>>>(l, out)));
}

}  // namespace

int32_t launch_embedding(const EmbeddingLaunch& a, hipStream_t stream) {
    const uint32_t lanes = row_lanes(a.dim);
    const Lookup l{a.table, (uint32_t)a.vocab, (uint32_t)a.dim, {a.ids, a.ids64}, a.n, a.scale, a.out_stride, lanes};
    const dim3 grid = grid_of(ceil_div(a.n, 256 / lanes));
    const bool vec = a.dim % 8 == 0 && on_vectors(a.out, a.n, a.out_stride, a.out_dtype) &&
                     (a.table.codes || on_vectors(a.table.data, a.vocab, a.table.stride, a.table.dtype));
    SLLM_BY_DTYPE(a.out_dtype, T, {
        if (vec)
            launch_lookup<true>(l, grid, static_cast<T*>(a.out), stream);
        else
            launch_lookup<false>(l, grid, static_cast<T*>(a.out), stream);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

namespace {

uint64_t align256(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

struct GradPlan {
    uint64_t windows, pitch, keys_bytes, bytes;
};

GradPlan plan_grad(uint64_t n, uint64_t dim) {
    GradPlan p;
    p.windows = ceil_div(n, kWindow);
    p.pitch = (dim + 7) / 8 * 8;
    p.keys_bytes = align256(n * 8);
    // two copies of the keys where they are merged, sums where runs can cross windows
    p.bytes = (n > kSortTile ? 2 : 1) * p.keys_bytes + (p.windows > 1 ? p.windows * 2 * p.pitch * 4 : 0);
    return p;
}

template <bool Vec, typename S, typename T>
int32_t launch_sums(const GradArgs& g, const EmbeddingGradLaunch& a, dim3 grid, hipStream_t stream) {
    T* grad = static_cast<T*>(a.grad);
    sum_runs<Vec, S, T><<<grid, 256, 0, stream>>>(g, static_cast<const S*>(a.dy), grad);
    SLLM_HIP(hipGetLastError());
    if (g.windows > 1) {
        // a frequent token's columns go to several CUs, each of which takes in only so much
        GradArgs j = g;
        j.lanes = std::min(g.lanes, 64u);
        j.chunks = (uint32_t)ceil_div(g.dim, j.lanes * 8);
        join_runs<Vec, T><<<(uint32_t)(ceil_div(g.windows, 256 / j.lanes) * j.chunks), 256, 0, stream>>>(j, grad);
        SLLM_HIP(hipGetLastError());
    }
    return SLLM_OK;
}

}  // namespace

uint64_t embedding_grad_workspace(uint64_t n_ids, uint64_t vocab, uint64_t dim) { return plan_grad(n_ids, dim).bytes; }

int32_t launch_embedding_grad(const EmbeddingGradLaunch& a, void* workspace, hipStream_t stream) {
    const GradPlan p = plan_grad(a.n, a.dim);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    uint64_t* keys = reinterpret_cast<uint64_t*>(ws);
    if (a.n) {
        const uint32_t tiles = (uint32_t)ceil_div(a.n, kSortTile);
        const Ids ids{a.ids, a.ids64};
        if (a.vocab < (1u << 22) - 1)
            sort_tiles<<<tiles, kSortTile, 0, stream>>>(ids, (uint32_t)a.n, (uint32_t)a.vocab, keys);
        else
            sort_tiles_wide<<<tiles, kSortTile, 0, stream>>>(ids, (uint32_t)a.n, (uint32_t)a.vocab, keys);
        SLLM_HIP(hipGetLastError());
        uint64_t* other = reinterpret_cast<uint64_t*>(ws + p.keys_bytes);
        for (uint64_t run = kSortTile; run < a.n; run *= kMergeRuns) {
            merge_runs<<<(uint32_t)ceil_div(a.n * kMergeRuns, 256), 256, 0, stream>>>(keys, (uint32_t)a.n, (uint32_t)run, other);
            SLLM_HIP(hipGetLastError());
            std::swap(keys, other);
        }
    }
    GradArgs g;
    g.keys = keys;
    g.n = (uint32_t)a.n, g.vocab = (uint32_t)a.vocab, g.dim = (uint32_t)a.dim;
    g.scale = a.scale;
    g.dy_stride = a.dy_stride, g.grad_stride = a.grad_stride;
    g.accumulate = a.accumulate;
    g.partial = reinterpret_cast<float*>(ws + (a.n > kSortTile ? 2 : 1) * p.keys_bytes);
    g.pitch = (uint32_t)p.pitch, g.windows = (uint32_t)p.windows;
    g.lanes = row_lanes(a.dim);
    g.chunks = (uint32_t)ceil_div(a.dim, g.lanes * 8);
    const uint64_t sums = ceil_div(p.windows, 256 / g.lanes) * g.chunks;
    const dim3 grid = grid_of(sums + (a.accumulate ? 0 : ceil_div(a.vocab, kZeroRows)));
    g.sum_blocks = (uint32_t)sums;
    const uint64_t size = element_bytes(a.grad_dtype), row_bytes = a.dim * size;
    const uint64_t steps = reinterpret_cast<uintptr_t>(a.grad) | row_bytes | (a.vocab > 1 ? a.grad_stride * size : 0);
    g.row_bytes = row_bytes;
    g.unit = steps % 16 == 0 ? 16 : steps % 4 == 0 ? 4 : 2;
    for (g.clear_lanes = 1; g.clear_lanes < 256 && g.clear_lanes < row_bytes / g.unit;) g.clear_lanes *= 2;
    const bool vec = a.dim % 8 == 0 && on_vectors(a.dy, a.n, a.dy_stride, a.dy_dtype) &&
                     on_vectors(a.grad, a.vocab, a.grad_stride, a.grad_dtype);
    SLLM_BY_DTYPE(a.dy_dtype, S, SLLM_BY_DTYPE(a.grad_dtype, T, return vec ? (launch_sums<true, S, T>(g, a, grid, stream))
                                                                          : (launch_sums<false, S, T>(g, a, grid, stream))));
    return SLLM_OK;
}

}  // namespace sllm
