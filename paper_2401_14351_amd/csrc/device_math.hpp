// Device helpers of the operators: element types and MX FP4 values.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "operators.hpp"

namespace sllm {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// An element as a 32-bit float (exact) and a float rounded to an element, to
// nearest even, overflow to infinity.
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
    return (T)v;
}

// On a lambda of a kernel: one that is not inlined takes what it captures, the
// accumulators among it, through memory.
#define SLLM_INLINE __attribute__((always_inline))

// Run F<T> for the element type of a dtype code.
#define SLLM_BY_DTYPE(dtype, T, ...)          \
    do {                                      \
        if ((dtype) == SLLM_DTYPE_F32) {      \
            using T = float;                  \
            __VA_ARGS__;                      \
        } else if ((dtype) == SLLM_DTYPE_F16) { \
            using T = _Float16;               \
            __VA_ARGS__;                      \
        } else {                              \
            using T = __bf16;                 \
            __VA_ARGS__;                      \
        }                                     \
    } while (0)

// Workgroups (of at most 1024 threads) in two dimensions where there are more than one
// can count, and which of them this one is.  A few more than asked for are launched.
inline dim3 grid_of(uint64_t blocks) {
    constexpr uint64_t kMost = 1 << 21;  // a dimension counts threads in 32 bits
    const uint64_t y = (blocks + kMost - 1) / kMost;
    return y <= 1 ? dim3((uint32_t)blocks) : dim3((uint32_t)((blocks + y - 1) / y), (uint32_t)y);
}
__device__ __forceinline__ uint32_t block_index() {
    return blockIdx.y ? blockIdx.y * gridDim.x + blockIdx.x : blockIdx.x;
}

// The scale operand of the conversion instructions: they take a float's
// exponent field alone, so a scale byte goes there as it is.  0 then means
// 2^-127 and 255 makes the results NaN, as the format has it.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace sllm
