// gfx950 kernels of root-mean-square norms, and of matrices in MX FP8.
#include <algorithm>

#include "common.hpp"
#include "device_math.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

namespace {

// Eight elements from column c, every Step-th, zeros past the end of the row.  Vec: the row
// starts on 16 bytes and ends on a multiple of eight columns, and they are neighbours.
template <bool Vec, typename T, int Step = 1>
struct Eight {
    static_assert(!Vec || Step == 1, "");
    T e[8];

    __device__ __forceinline__ void load(const T* row, uint64_t c, uint64_t cols) {
        if (Vec) {
            u32x4 raw[sizeof(T) / 2] = {};
            if (c < cols)
#pragma unroll
                for (uint32_t i = 0; i < sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const u32x4*>(row + c)[i];
            __builtin_memcpy(e, raw, sizeof e);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c + i * Step < cols ? row[c + i * Step] : (T)0.0f;
        }
    }
    // The same without a condition on a load, where the compiler waits for those one by one: in
    // the gradients, of 16 bits (8191 x 5121 in bf16: 334 us, 112 so; float 136, 147 so; the norm
    // itself 90 and 163, since what is past the end is then read too).
    __device__ __forceinline__ void load_all(const T* row, uint64_t c, uint64_t cols) {
        if (Vec || sizeof(T) == 4) return load(row, c, cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const T v = row[min(c + i * Step, cols - 1)];
            e[i] = c + i * Step < cols ? v : (T)0.0f;
        }
    }
    __device__ __forceinline__ void store(T* row, uint64_t c, uint64_t cols) const {
        if (Vec) {
            u32x4 raw[sizeof(T) / 2];
            __builtin_memcpy(raw, e, sizeof e);
            if (c < cols)
#pragma unroll
                for (uint32_t i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<u32x4*>(row + c)[i] = raw[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i * Step < cols) row[c + i * Step] = e[i];
        }
    }
};

// The gain, of any type.
template <bool Vec, int Step, typename G>
__device__ __forceinline__ void load_floats(const G* from, uint64_t c, uint64_t cols, float (&g)[8]) {
    Eight<Vec, G, Step> v;
    v.load(from, c, cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = to_f32(v.e[i]);
}
template <bool Vec, int Step>
__device__ __forceinline__ void load_gain(const void* gain, uint32_t dtype, uint64_t c, uint64_t cols, float (&g)[8]) {
    SLLM_BY_DTYPE(dtype, G, load_floats<Vec, Step>(static_cast<const G*>(gain), c, cols, g));
}

// The sum over the `Lanes` threads of a row, in all of them: the same order on every call.
template <int Lanes, typename S>
__device__ __forceinline__ S row_sum(S x, S* waves) {
#pragma unroll
    for (int d = Lanes < 64 ? Lanes / 2 : 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    if constexpr (Lanes > 64) {
        if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < Lanes / 64; ++w) x += waves[w];
        __syncthreads();
    }
    return x;
}

template <int Ctrl>
__device__ __forceinline__ uint32_t quad(uint32_t x) {
    return __builtin_amdgcn_mov_dpp(x, Ctrl, 0xF, 0xF, true);
}

// A double as the float that rounds as it does to anything of fewer bits: cut off, its last
// bit set where something was.
__device__ __forceinline__ float to_odd(double d) {
    uint64_t bits = __builtin_bit_cast(uint64_t, d);
    constexpr uint64_t kRest = (1ull << 29) - 1;
    bits = (bits & ~kRest) | (bits & kRest ? 1ull << 29 : 0);
    return (float)__builtin_bit_cast(double, bits);
}

// Eight values of a block of 32, which four neighbouring lanes hold, in MX FP8: codes, and
// the block's scale byte.  The scale is the smallest power of two whose 448-fold, the
// largest E4M3 value, is not below the block's largest magnitude: nothing saturates.
__device__ __forceinline__ u32x2 to_fp8(const float (&v)[8], uint32_t& scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffff);
    top = max(top, quad<0xB1>(top));  // lanes 1 0 3 2
    top = max(top, quad<0x4E>(top));  // lanes 2 3 0 1
    const uint32_t e = top >> 23;
    if (e == 255) {  // an infinity or a NaN
        scale = 255;
        return u32x2{0, 0};
    }
    const uint32_t up = e + ((top & 0x7fffff) > 0x600000);  // above 1.75 times a power of two
    scale = up > 8 ? up - 8 : 0;
    const float f = __uint_as_float((254 - scale) << 23);  // a power of two: exact but for what rounds to zero
    u32x2 out;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * f, v[4 * i + 1] * f, 0, false);
        out[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * f, v[4 * i + 3] * f, w, true);
    }
    return out;
}

struct NormArgs {
    const void *x, *residual, *gain;
    uint64_t x_stride, residual_stride, rows, cols;
    uint32_t gain_dtype;
    float eps;
    void *h, *y;
    uint64_t h_stride, y_stride;
    float* inverse;
    uint8_t *codes, *scales;  // y in MX FP8
};

// h = x + residual, rounded; y = h / sqrt(mean h^2 + eps) * gain.  Bound by memory: x and
// the residual are read once, h and y written once (8191 x 5120 in bf16, 336 MB: 66 us, 5.1
// TB/s; 4096 x 8192 to MX FP8 57 to 65; a row of 4096 3 us, a launch and two reads in turn).  `Lanes` threads take a row and keep
// up to `Held` times eight of its columns each; longer rows are read again, by the threads
// that have written them.
//
// The sum of squares is held in 64 bits: those of 32-bit elements may leave 32.  In MX FP8
// the whole norm is, up to its rounding: an element next to the middle of two of the few
// values there are then goes to the one that is nearer.
template <typename T, int Lanes, int Held, bool Vec, bool Mx8>
__global__ __launch_bounds__(Lanes < 256 ? 256 : Lanes) void rms_norm(NormArgs a) {
    typedef typename std::conditional<Mx8, double, float>::type S;
    __shared__ double waves[16];
    constexpr uint32_t kThreads = Lanes < 256 ? 256 : Lanes;
    const uint64_t row = (uint64_t)block_index() * (kThreads / Lanes) + threadIdx.x / Lanes;
    if (row >= a.rows) return;  // all threads of a row, which alone meet
    const uint32_t l = threadIdx.x % Lanes;
    constexpr int kStep = Vec || Mx8 ? 1 : Lanes;
    const uint32_t l0 = kStep == 1 ? l * 8 : l;  // this thread's first column of 8 Lanes
    const T* const x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* const residual = static_cast<const T*>(a.residual) + row * a.residual_stride;
    T* const h = static_cast<T*>(a.h) + row * a.h_stride;
    const uint64_t blocks = (a.cols + 31) / 32, pitch = (blocks + 15) / 16 * 16;
    const uint64_t end = Mx8 ? pitch * 32 : a.cols;

    const auto load = [&](uint64_t c, Eight<Vec, T, kStep>& v) SLLM_INLINE {
        v.load(x, c, a.cols);
        if (a.residual) {
            Eight<Vec, T, kStep> r;
            r.load(residual, c, a.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) v.e[i] = from_f32<T>(to_f32(v.e[i]) + to_f32(r.e[i]));
        }
    };
    double sum = 0;
    const auto add = [&](const Eight<Vec, T, kStep>& v) SLLM_INLINE {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (double)to_f32(v.e[i]) * (double)to_f32(v.e[i]);
    };
    S f = 0;
    const auto write = [&](uint64_t c, const Eight<Vec, T, kStep>& v, const float (&g)[8]) SLLM_INLINE {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (Mx8)
                y[i] = to_odd((S)to_f32(v.e[i]) * f * (S)g[i]);
            else
                y[i] = to_f32(v.e[i]) * f * g[i];
        }
        if constexpr (Mx8) {
            const uint64_t b = c / 32;
            if (c >= a.cols)  // what the padding of a block would make of an f that is no number
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = 0;
            else if (!Vec)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = c + i < a.cols ? y[i] : 0;
            uint32_t scale;
            const u32x2 codes = to_fp8(y, scale);
            if (b < blocks) *reinterpret_cast<u32x2*>(a.codes + row * blocks * 32 + c) = codes;
            if (c % 32 == 0 && b < pitch) a.scales[row * pitch + b] = b < blocks ? scale : 0;
        } else {
            Eight<Vec, T, kStep> o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o.e[i] = from_f32<T>(y[i]);
            o.store(static_cast<T*>(a.y) + row * a.y_stride, c, a.cols);
        }
    };
    const auto finish = [&]() SLLM_INLINE {
        sum = row_sum<Lanes>(sum, waves);
        f = (S)(1 / sqrt(sum / (double)a.cols + a.eps));
        if (a.inverse && l == 0) a.inverse[row] = (float)f;
    };
    if constexpr (Held > 0) {
        Eight<Vec, T, kStep> v[Held];
        float g[Held][8];
#pragma unroll
        for (int i = 0; i < Held; ++i) load(i * Lanes * 8 + l0, v[i]);
#pragma unroll
        for (int i = 0; i < Held; ++i) {
            load_gain<Vec, kStep>(a.gain, a.gain_dtype, i * Lanes * 8 + l0, a.cols, g[i]);
            add(v[i]);
            if (a.residual) v[i].store(h, i * Lanes * 8 + l0, a.cols);
        }
        finish();
#pragma unroll
        for (int i = 0; i < Held; ++i)
            if (i * Lanes * 8 + l0 < end) write(i * Lanes * 8 + l0, v[i], g[i]);
    } else {
        for (uint64_t c = l0; c < a.cols; c += Lanes * 8) {
            Eight<Vec, T, kStep> v;
            load(c, v);
            add(v);
            if (a.residual) v.store(h, c, a.cols);
        }
        finish();
        for (uint64_t c = l0; c < end; c += Lanes * 8) {
            Eight<Vec, T, kStep> v;
            float g[8];
            v.load(a.residual ? h : x, c, a.cols);
            load_gain<Vec, kStep>(a.gain, a.gain_dtype, c, a.cols, g);
            write(c, v, g);
        }
    }
}

struct NormGradArgs {
    const void *dy, *dh, *h, *gain;
    uint64_t dy_stride, dh_stride, h_stride, rows, cols;
    uint32_t gain_dtype;
    const float* inverse;
    void* dx;
    uint64_t dx_stride;
    float* parts;   // slots x cols: the gain's gradient, of the rows a slot has had
    uint32_t slots;
};

// With f = 1 / sqrt(mean h^2 + eps) and s = dy gain: dx = dh + f (s - h f^2 mean(s h)), and
// the gain's gradient is the sum over rows of dy h f.  h only comes with its f, as the norm,
// whose elements are of ordinary size whatever the row's are.  Bound by memory (8191 x 5120 in
// bf16, 336 MB: 63 to 74 us; 16384 x 8192 161, 5.0 TB/s).  `Lanes` threads
// take a row at a time, of every `slots`-th row, and keep their columns' sums; where a row
// is too long for that the sums are kept in memory.  Short rows are taken by a workgroup side
// by side, which adds up their sums.
template <typename T, int Lanes, int Held, bool Vec>
__global__ __launch_bounds__(Lanes < 256 ? 256 : Lanes) void rms_norm_grad(NormGradArgs a) {
    __shared__ float waves[16];
    constexpr uint32_t kThreads = Lanes < 256 ? 256 : Lanes;
    constexpr uint32_t kSide = Held == 1 ? kThreads / Lanes : 1, kSlots = kThreads / Lanes / kSide;
    __shared__ float joined[kSide > 1 ? 3 : 1][kSide > 1 ? Lanes * 8 : 1];
    const uint32_t slot = blockIdx.x * kSlots + threadIdx.x / (Lanes * kSide), l = threadIdx.x % Lanes, side = threadIdx.x / Lanes % kSide;
    if (slot >= a.slots) return;
    constexpr int kStep = Vec ? 1 : Lanes;
    const uint32_t l0 = kStep == 1 ? l * 8 : l;  // this thread's first column of 8 Lanes
    float* const part = a.parts + (uint64_t)slot * a.cols;
    const auto dx_of = [&](const Eight<Vec, T, kStep>& dy, const Eight<Vec, T, kStep>& h, const Eight<Vec, T, kStep>& dh, const float (&g)[8], float f, float along) SLLM_INLINE {
        Eight<Vec, T, kStep> dx;
#pragma unroll
        for (int i = 0; i < 8; ++i) dx.e[i] = from_f32<T>(to_f32(dh.e[i]) + f * (to_f32(dy.e[i]) * g[i] - to_f32(h.e[i]) * f * along));
        return dx;
    };
    const auto load_dh = [&](uint64_t row, uint64_t c) SLLM_INLINE {
        Eight<Vec, T, kStep> dh;
#pragma unroll
        for (int i = 0; i < 8; ++i) dh.e[i] = (T)0.0f;
        if (a.dh) dh.load_all(static_cast<const T*>(a.dh) + row * a.dh_stride, c, a.cols);
        return dh;
    };
    if constexpr (Held > 0) {
        float g[Held][8], sums[Held][8] = {};
#pragma unroll
        for (int i = 0; i < Held; ++i) load_gain<Vec, kStep>(a.gain, a.gain_dtype, i * Lanes * 8 + l0, a.cols, g[i]);
        for (uint64_t row = (uint64_t)slot * kSide + side; row < a.rows; row += (uint64_t)a.slots * kSide) {
            const float f = a.inverse[row];
            Eight<Vec, T, kStep> dy[Held], h[Held], dh[Held];
#pragma unroll
            for (int i = 0; i < Held; ++i) {
                dy[i].load_all(static_cast<const T*>(a.dy) + row * a.dy_stride, i * Lanes * 8 + l0, a.cols);
                h[i].load_all(static_cast<const T*>(a.h) + row * a.h_stride, i * Lanes * 8 + l0, a.cols);
                dh[i] = load_dh(row, i * Lanes * 8 + l0);
            }
            float dot = 0;
#pragma unroll
            for (int i = 0; i < Held; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = to_f32(dy[i].e[e]) * (to_f32(h[i].e[e]) * f);
                    dot += d * g[i][e];
                    sums[i][e] += d;
                }
            const float along = row_sum<Lanes>(dot, waves) / (float)a.cols;
#pragma unroll
            for (int i = 0; i < Held; ++i)
                dx_of(dy[i], h[i], dh[i], g[i], f, along).store(static_cast<T*>(a.dx) + row * a.dx_stride, i * Lanes * 8 + l0, a.cols);
        }
        if constexpr (kSide > 1) {
            // rows of a wave, then the waves
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int d = Lanes; d < 64; d *= 2) sums[0][e] += __shfl_xor(sums[0][e], d);
                if (threadIdx.x >= 64 && threadIdx.x % 64 < Lanes) joined[threadIdx.x / 64 - 1][l * 8 + e] = sums[0][e];
            }
            __syncthreads();
            if (side) return;
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int w = 0; w < 3; ++w) sums[0][e] += joined[w][l * 8 + e];
        }
#pragma unroll
        for (int i = 0; i < Held; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i * Lanes * 8 + l0 + e * kStep < a.cols) part[i * Lanes * 8 + l0 + e * kStep] = sums[i][e];
    } else {
        for (uint64_t row = slot; row < a.rows; row += a.slots) {
            const float f = a.inverse[row];
            const T *dy_row = static_cast<const T*>(a.dy) + row * a.dy_stride, *h_row = static_cast<const T*>(a.h) + row * a.h_stride;
            float dot = 0;
            for (uint64_t c = l0; c < a.cols; c += Lanes * 8) {
                Eight<Vec, T, kStep> dy, h;
                float g[8];
                dy.load_all(dy_row, c, a.cols);
                h.load_all(h_row, c, a.cols);
                load_gain<Vec, kStep>(a.gain, a.gain_dtype, c, a.cols, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = to_f32(dy.e[e]) * (to_f32(h.e[e]) * f);
                    dot += d * g[e];
                    if (c + e * kStep < a.cols) part[c + e * kStep] = (row == slot ? 0.0f : part[c + e * kStep]) + d;
                }
            }
            const float along = row_sum<Lanes>(dot, waves) / (float)a.cols;
            for (uint64_t c = l0; c < a.cols; c += Lanes * 8) {
                Eight<Vec, T, kStep> dy, h;
                float g[8];
                dy.load_all(dy_row, c, a.cols);
                h.load_all(h_row, c, a.cols);
                load_gain<Vec, kStep>(a.gain, a.gain_dtype, c, a.cols, g);
                dx_of(dy, h, load_dh(row, c), g, f, along).store(static_cast<T*>(a.dx) + row * a.dx_stride, c, a.cols);
            }
        }
    }
}

// The slots' sums, in their order: 32 runs of slots side by side, then those (512 x 5120: 4.0 us).
template <typename G>
__global__ __launch_bounds__(1024) void join_gain(const float* parts, uint32_t slots, uint64_t cols, G* out) {
    constexpr uint32_t kRuns = 32, kCols = 32;
    __shared__ float sums[kRuns][kCols];
    const uint32_t l = threadIdx.x % kCols, run = threadIdx.x / kCols;
    const uint64_t c = (uint64_t)block_index() * kCols + l;
    float sum = 0;
    if (c < cols) {
        const uint32_t end = (uint64_t)slots * (run + 1) / kRuns;
#pragma unroll 8
        for (uint32_t s = (uint64_t)slots * run / kRuns; s < end; ++s) sum += parts[s * cols + c];
    }
    sums[run][l] = sum;
    __syncthreads();
    if (run || c >= cols) return;
#pragma unroll
    for (uint32_t i = 1; i < kRuns; ++i) sum += sums[i][l];
    out[c] = from_f32<G>(sum);
}

bool vector_rows(const void* p, uint64_t stride, uint64_t rows, uint64_t cols, uint64_t size) {
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols % 8 == 0 && (rows <= 1 || stride * size % 16 == 0));
}

// As few threads as hold a row: a sum within a wave is done sooner than across waves, and what
// is held in vain costs registers (in bf16, 2^25 elements, us: rows of 128 by 16 threads 25, by
// 64 81; 512 by 64 threads and one load each 24, with four 41; 1024 by 64 26, by 256 50; 2048 25
// and 30; 4096 with two loads 24, with four 28; 8192 with four 25, read twice by 1024 threads 30;
// 16384 by 1024 23.5, read twice 25.5; 32768 held by 1024 32.5, read twice 29).  One wave a row
// leaves CUs empty where rows are few, from 1025 columns on.
template <typename T, bool Vec, bool Mx8>
void launch_rows(const NormArgs& a, hipStream_t stream) {
    if constexpr (!Mx8) {
        if (a.cols <= 128) return rms_norm<T, 16, 1, Vec, Mx8><<<grid_of(ceil_div(a.rows, 16)), 256, 0, stream>>>(a);
    }
    if (a.cols <= 512)
        rms_norm<T, 64, 1, Vec, Mx8><<<grid_of(ceil_div(a.rows, 4)), 256, 0, stream>>>(a);
    else if (a.cols <= 1024 || (a.cols <= 2048 && a.rows >= 1024))
        rms_norm<T, 64, 4, Vec, Mx8><<<grid_of(ceil_div(a.rows, 4)), 256, 0, stream>>>(a);
    else if (a.cols <= 4096)
        rms_norm<T, 256, 2, Vec, Mx8><<<grid_of(a.rows), 256, 0, stream>>>(a);
    else if (a.cols <= 8192)
        rms_norm<T, 256, 4, Vec, Mx8><<<grid_of(a.rows), 256, 0, stream>>>(a);
    else if (a.cols <= 16384)
        rms_norm<T, 1024, 2, Vec, Mx8><<<grid_of(a.rows), 1024, 0, stream>>>(a);
    else
        rms_norm<T, 1024, 0, Vec, Mx8><<<grid_of(a.rows), 1024, 0, stream>>>(a);
}

template <typename T, bool Vec>
void launch_grad_rows(const NormGradArgs& a, hipStream_t stream) {
    if (a.cols <= 128)
        rms_norm_grad<T, 16, 1, Vec><<<dim3(a.slots), 256, 0, stream>>>(a);
    else if (a.cols <= 512)
        rms_norm_grad<T, 64, 1, Vec><<<dim3(a.slots), 256, 0, stream>>>(a);
    else if (a.cols <= 2048)
        rms_norm_grad<T, 64, 4, Vec><<<dim3((uint32_t)ceil_div(a.slots, 4)), 256, 0, stream>>>(a);
    else if (a.cols <= 4096)
        rms_norm_grad<T, 256, 2, Vec><<<dim3(a.slots), 256, 0, stream>>>(a);
    else if (a.cols <= 8192)
        rms_norm_grad<T, 512, 2, Vec><<<dim3(a.slots), 512, 0, stream>>>(a);
    else if (a.cols <= 16384)
        rms_norm_grad<T, 1024, 2, Vec><<<dim3(a.slots), 1024, 0, stream>>>(a);
    else
        rms_norm_grad<T, 1024, 0, Vec><<<dim3(a.slots), 1024, 0, stream>>>(a);
}

// Rows of the workspace, one for the rows that a slot of workgroups takes in turn, or side by
// side: as many as the GPU holds at once, since more have to be written and joined.  (2^27
// elements in bf16, 805 MB, us: 1024 columns with 256, 1024, 2048 and 4096 slots 733, 215, 156 and
// 174; 4096 with 256, 512, 768 and 2048 213, 153, 161 and 176; 8192 165, 161, 172 and 193, by 256
// threads that hold twice as much 184, 165, 180 and 193; 16384 160, 170, 184 and 252.)
uint32_t grad_slots(uint64_t rows, uint64_t cols) {
    const uint64_t most = cols <= 2048 ? 2048 : cols <= 8192 ? 512 : 256, side = cols <= 128 ? 16 : cols <= 512 ? 4 : 1;
    return (uint32_t)std::min<uint64_t>(ceil_div(rows, side), most);
}

// x in MX FP8: as mx_quantize is for MX FP4.
template <bool Vec, typename T>
__global__ __launch_bounds__(256) void mx8_quantize(const T* src, uint64_t stride, uint64_t rows, uint64_t cols, uint32_t lanes, uint8_t* codes,
                                                    uint8_t* scales) {
    const uint64_t row = (uint64_t)block_index() * (256 / lanes) + threadIdx.x / lanes;
    if (row >= rows) return;
    const uint64_t blocks = (cols + 31) / 32, pitch = (blocks + 15) / 16 * 16;
    for (uint64_t i = threadIdx.x % lanes; i < pitch * 4; i += lanes) {
        const uint64_t b = i / 4, c = i * 8;
        Eight<Vec, T> e;
        e.load(src + row * stride, c, cols);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = to_f32(e.e[j]);
        uint32_t scale;
        const u32x2 out = to_fp8(v, scale);
        if (b < blocks) *reinterpret_cast<u32x2*>(codes + row * blocks * 32 + c) = out;
        if (i % 4 == 0) scales[row * pitch + b] = b < blocks ? scale : 0;
    }
}

template <bool Vec, typename T>
__global__ __launch_bounds__(256) void mx8_dequantize(const uint8_t* codes, const uint8_t* scales, uint64_t rows, uint64_t cols, T* out,
                                                      uint64_t stride) {
    const uint64_t vectors = (cols + 7) / 8, blocks = (cols + 31) / 32, pitch = (blocks + 15) / 16 * 16;
    const uint64_t i = (uint64_t)block_index() * 256 + threadIdx.x, row = i / vectors, c = i % vectors * 8;
    if (row >= rows) return;
    const u32x2 v = *reinterpret_cast<const u32x2*>(codes + row * blocks * 32 + c);
    const uint32_t s = scales[row * pitch + c / 32];
    float f[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        f[4 * j] = __builtin_amdgcn_cvt_f32_fp8(v[j], 0);
        f[4 * j + 1] = __builtin_amdgcn_cvt_f32_fp8(v[j], 1);
        f[4 * j + 2] = __builtin_amdgcn_cvt_f32_fp8(v[j], 2);
        f[4 * j + 3] = __builtin_amdgcn_cvt_f32_fp8(v[j], 3);
    }
    Eight<Vec, T> o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o.e[j] = from_f32<T>(s == 255 ? __builtin_nanf("") : __builtin_ldexpf(f[j], (int)s - 127));
    o.store(out + row * stride, c, cols);
}

}  // namespace

int32_t launch_rms_norm(const NormLaunch& n, hipStream_t stream) {
    const uint64_t size = n.dtype == SLLM_DTYPE_F32 ? 4 : 2;
    const bool vec = n.cols % 8 == 0 && vector_rows(n.x, n.x_stride, n.rows, n.cols, size) &&
                     vector_rows(n.residual, n.residual_stride, n.rows, n.cols, size) && vector_rows(n.h, n.h_stride, n.rows, n.cols, size) &&
                     vector_rows(n.y, n.y_stride, n.rows, n.cols, size) && vector_rows(n.gain, 0, 1, n.cols, 4);
    const NormArgs a{n.x, n.residual, n.gain, n.x_stride, n.residual_stride, n.rows, n.cols, n.gain_dtype, n.eps,
                     n.h, n.y, n.h_stride, n.y_stride, n.inverse, n.codes, n.scales};
    SLLM_BY_DTYPE(n.dtype, T, {
        if (n.codes)
            vec ? launch_rows<T, true, true>(a, stream) : launch_rows<T, false, true>(a, stream);
        else
            vec ? launch_rows<T, true, false>(a, stream) : launch_rows<T, false, false>(a, stream);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

uint64_t rms_norm_grad_workspace(uint64_t rows, uint64_t cols) { return (uint64_t)grad_slots(rows, cols) * cols * 4; }

int32_t launch_rms_norm_grad(const NormGradLaunch& n, void* workspace, hipStream_t stream) {
    const uint64_t size = n.dtype == SLLM_DTYPE_F32 ? 4 : 2;
    const bool vec = n.cols % 8 == 0 && vector_rows(n.dy, n.dy_stride, n.rows, n.cols, size) && vector_rows(n.dh, n.dh_stride, n.rows, n.cols, size) &&
                     vector_rows(n.h, n.h_stride, n.rows, n.cols, size) && vector_rows(n.dx, n.dx_stride, n.rows, n.cols, size) &&
                     vector_rows(n.gain, 0, 1, n.cols, 4);
    const NormGradArgs a{n.dy, n.dh, n.h, n.gain, n.dy_stride, n.dh_stride, n.h_stride, n.rows, n.cols, n.gain_dtype, n.inverse,
                         n.dx, n.dx_stride, static_cast<float*>(workspace), grad_slots(n.rows, n.cols)};
    if (n.rows) {
        SLLM_BY_DTYPE(n.dtype, T, { vec ? launch_grad_rows<T, true>(a, stream) : launch_grad_rows<T, false>(a, stream); });
        SLLM_HIP(hipGetLastError());
    }
    SLLM_BY_DTYPE(n.gain_dtype, G,
                  (join_gain<G><<<grid_of(ceil_div(n.cols, 32)), 1024, 0, stream>>>(a.parts, a.slots, n.cols, static_cast<G*>(n.dgain))));
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

int32_t launch_mx8_quantize(const sllm_matrix& src, const sllm_mx& dst, hipStream_t stream) {
    const uint32_t lanes = mx_scale_pitch(src.cols) * 4 >= 256 ? 256 : 64;
    const dim3 grid = grid_of(ceil_div(src.rows, 256 / lanes));
    const bool vec = vector_rows(src.data, src.stride, src.rows, src.cols, src.dtype == SLLM_DTYPE_F32 ? 4 : 2);
    uint8_t *codes = static_cast<uint8_t*>(dst.codes), *scales = static_cast<uint8_t*>(dst.scales);
    SLLM_BY_DTYPE(src.dtype, T, {
        const T* x = static_cast<const T*>(src.data);
        (vec ? mx8_quantize<true, T> : mx8_quantize<false, T>)<<<grid, 256, 0, stream>>>(x, src.stride, src.rows, src.cols, lanes, codes, scales);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

int32_t launch_mx8_dequantize(const sllm_mx& src, const sllm_matrix& dst, hipStream_t stream) {
    const dim3 grid = grid_of(ceil_div(src.rows * ceil_div(src.cols, 8), 256));
    const bool vec = vector_rows(dst.data, dst.stride, dst.rows, dst.cols, dst.dtype == SLLM_DTYPE_F32 ? 4 : 2);
    const uint8_t *codes = static_cast<const uint8_t*>(src.codes), *scales = static_cast<const uint8_t*>(src.scales);
    SLLM_BY_DTYPE(dst.dtype, T, {
        T* out = static_cast<T*>(dst.data);
        (vec ? mx8_dequantize<true, T> : mx8_dequantize<false, T>)<<<grid, 256, 0, stream>>>(codes, scales, src.rows, src.cols, out, dst.stride);
    });
    SLLM_HIP(hipGetLastError());
    return SLLM_OK;
}

}  // namespace sllm
