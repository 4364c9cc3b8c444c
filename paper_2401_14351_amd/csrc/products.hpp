// What the kernels of products with an MX FP4 weight share.
#pragma once

#include "device_math.hpp"

namespace sllm {

constexpr uint32_t kTileRows = 4;  // of tiles that neighbouring workgroups share
constexpr uint32_t kWideStep = 64;   // depth of a stage

// Where a product's sums go: m x cols, or, where the depth is split over
// workgroups (blockIdx.y), a 32-bit matrix per split, one after another.
struct OutArgs {
    uint64_t m, cols, stride;
    uint64_t split_stride;  // elements from one split's matrix to the next
    uint32_t vector;        // rows start on 16 bytes
};

// x (m x depth) in float16, or (parts of it one after another along a row) in bfloat16
struct WideArgs {
    const uint16_t* x;
    uint64_t m, depth;       // of a part
    uint64_t x_stride, part_stride;
    uint32_t parts, steps;   // steps of a part, an even number
    const uint32_t* ranges;  // of the rows of a float16 x; null: each workgroup finds those of its piece
    const u32x4* w_codes;
    const uint8_t* w_scales;
    uint64_t w_rows, w_blocks, w_scale_pitch;
    uint32_t tiles_m, tiles_j;
    OutArgs out_args;
};

// What lanes past the end of the depth load.
static __device__ const u32x4 kZeroVector = {0, 0, 0, 0};

// Its address, as a value the compiler cannot tell: a lane's choice between it
// and its own address then is a select, not a branch with a load on either side.
__device__ __forceinline__ const void* zero_vector() {
    uintptr_t p = reinterpret_cast<uintptr_t>(&kZeroVector);
    asm("" : "+v"(p));
    return reinterpret_cast<const void*>(p);
}

// A workgroup's LDS, by a variable and an offset into it.  The compiler keeps track
// of which variable an access is to, and then waits for no load into another
// before it, if the address space is known from the start and the address is a
// short sum: offsets of a lane go through opaque().
__device__ __forceinline__ uint32_t opaque(uint32_t v) {
    asm("" : "+v"(v));
    return v;
}
typedef __attribute__((address_space(3))) uint8_t lds_u8;

template <typename V>
__device__ __forceinline__ V lds_read(const uint8_t* p, uint32_t at) {
    return *reinterpret_cast<const __attribute__((address_space(3))) V*>((const lds_u8*)p + at);
}

template <typename V>
__device__ __forceinline__ void lds_write(uint8_t* p, uint32_t at, V v) {
    *reinterpret_cast<__attribute__((address_space(3))) V*>((lds_u8*)p + at) = v;
}

// 16 bytes a lane straight to LDS: p + at is the same in all lanes of the wave,
// and lane l's go to 16 l bytes past it.
__device__ __forceinline__ void load_to_lds(const void* from, uint8_t* p, uint32_t at) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)((lds_u8*)p + at), 16, 0, 0);
}

// Four bytes a lane, lane l's to 4 l past p + at.
__device__ __forceinline__ void load_word_to_lds(const void* from, uint8_t* p, uint32_t at) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)((lds_u8*)p + at), 4, 0, 0);
}

// Lanes of a wave see what each other wrote to LDS.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// All but the last N loads of this wave have landed, those to LDS included, and
// its reads and writes of LDS are done.  The counts are in the operand's fields:
// vmcnt in bits 3:0 and 15:14, expcnt (not waited for) in 6:4, lgkmcnt in 11:8.
template <int N>
__device__ __forceinline__ void wait_but_loads() {
    static_assert(N < 64, "");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
}

// A barrier that waits for nothing else: __syncthreads would wait for all loads.
__device__ __forceinline__ void barrier() {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The tile of a workgroup.  Workgroups go to the eight XCDs in turn; each XCD
// takes a run of tiles of its own, four rows of tiles at a time, so that its
// 32 CUs work on a patch of the output and find each other's operands in its L2.
struct Tile {
    uint32_t m, j;
};
__device__ __forceinline__ Tile tile_of(uint32_t block, uint32_t tiles_m, uint32_t tiles_j) {
    const uint32_t tiles = tiles_m * tiles_j, xcd = block % 8, q = tiles / 8, rest = tiles % 8;
    const uint32_t i = xcd * q + min(xcd, rest) + block / 8;
    const uint32_t group = i / (kTileRows * tiles_j), in = i % (kTileRows * tiles_j);
    const uint32_t rows = min(kTileRows, tiles_m - group * kTileRows);
    return {group * kTileRows + in % rows, in / rows};
}

// Where chunk c (of eight, 16 bytes each) of row r of a tile lies in LDS.  Rows
// are 128 bytes: eight lanes load one, whole, and a load straight to LDS puts
// lane l's bytes at 16 l, so the order of a row's chunks is chosen by what each
// lane loads.  It changes every other row, so that 16 rows read in one column of
// chunks, by 16 neighbouring lanes, are in all banks once.  chunk_at(r, c ^ s) is chunk_at(r, c) ^ 16 s.
__device__ __forceinline__ uint32_t chunk_at(uint32_t r, uint32_t c) { return r * 128 + (c ^ (r >> 1 & 7)) * 16; }

// The same for rows of 64 bytes, four chunks: four rows are in all banks once.
__device__ __forceinline__ uint32_t short_chunk_at(uint32_t r, uint32_t c) { return r * 64 + (c ^ (r >> 2 & 3)) * 16; }

typedef int i32x8 __attribute__((ext_vector_type(8)));

// A block of codes as an operand of the scaled matrix instruction, whose other
// four registers 4-bit elements do not use.
__device__ __forceinline__ i32x8 fragment(u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }

// The leading eight bits of f as a bfloat16, and f less those: two or three of
// these in turn are all of a float16 or a float.  An infinity or a NaN is whole
// in the first and leaves zero.
__device__ __forceinline__ uint32_t leading_bf16(float& f) {
    const uint32_t bits = __float_as_uint(f);
    const bool finite = (bits & 0x7f800000) != 0x7f800000;
    f = finite ? f - __uint_as_float(bits & 0xffff0000) : 0.0f;
    // a NaN whose payload is all in the lower half must not become an infinity
    return finite || !(bits & 0x7fffff) ? bits >> 16 : 0x7fc0;
}

// Eight codes as bfloat16 or float16.
template <typename X = __bf16>
__device__ __forceinline__ u32x4 expand8(uint32_t codes, float scale) {
    u32x4 v;
    if constexpr (__is_same(X, __bf16)) {
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    } else {
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3));
    }
    return v;
}

// 16 of the depth by 32 columns and 32 rows.
template <typename X>
__device__ __forceinline__ f32x16 product(u32x4 w, u32x4 x, f32x16 acc) {
    if constexpr (__is_same(X, __bf16))
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), acc, 0, 0, 0);
}

// An x in float16 is multiplied in float16, W times 2^kHalfShift and x's rows times a
// power of two each, so that every operand is zero or a normal number.  The matrix
// instruction adds products of a subnormal (below 2^-14) as if it were 2^-14 and drops
// what is 24 bits under that, of the sum so far too: with subnormals let in, sums of small
// products were off by up to 12 times what 32 bits allow.
//   * Blocks of W whose scale is not 2^-21 to 2^5 (values of 2^-22 to 192), other than
//     zeros, are left out, their stages marked, and added afterwards in bfloat16, x in
//     two parts.
//   * A row of x is multiplied by up to 2^10, which makes 2^-24, the smallest element, a
//     normal number, but by no more than its largest element allows; a kernel before, or
//     where that is quicker the workgroup itself, finds both.  Where a row has elements
//     more than 2^29 apart, or an infinity or a NaN, its workgroups take all stages in
//     bfloat16.
// 4096 x 8192 by 8192 takes 507 us (a bfloat16 x 410), 518 with a block left out in every
// tile, 2100 where every tile has such a row or leaves all of W out; 64 rows by 4096 x
// 4096 17.3 (13.6).
constexpr int kHalfShift = 8;
constexpr uint32_t kHalfScale = 127 - 21, kHalfScales = 27;

// A block's scale for its values in float16, times 2^kHalfShift.  A block of zeros may
// have any scale: those that the sum would make infinite stay finite, and zeros zeros.
__device__ __forceinline__ float half_scale(uint32_t byte) { return mx_scale(min(byte, 254u - kHalfShift) + kHalfShift); }

// Whether a block, or some of its codes, is left out.
__device__ __forceinline__ bool beyond_half(uint32_t scale, uint32_t codes) {
    return (scale - kHalfScale >= kHalfScales) & ((scale == 255) | ((codes & 0x77777777) != 0));
}

// Stages of which a workgroup has left something out, a bit each; those of a greater
// depth share the bits, and nothing is then added for most of them.
constexpr uint32_t kMarkWords = 64;
__device__ __forceinline__ void mark_stage(uint32_t* marks, uint32_t t) {
    if ((threadIdx.x & 63) == 0) atomicOr(&marks[t / 32 % kMarkWords], 1u << t % 32);
}
__device__ __forceinline__ bool marked(const uint32_t* marks, uint32_t t) { return marks[t / 32 % kMarkWords] >> t % 32 & 1; }

// A row's range: the bits of its largest magnitude, and above them those of its smallest
// but zero, less one (all ones where it is all zeros).
struct RowRange {
    uint32_t top = 0, bottom = 0xffff;

    __device__ __forceinline__ void add(u32x4 v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t size = v[i / 2] >> i % 2 * 16 & 0x7fff;
            top = max(top, size);
            bottom = min(bottom, (size - 1) & 0xffff);
        }
    }
    // Of `lanes` neighbours, a power of two.
    __device__ __forceinline__ void join(int lanes) {
        for (int d = lanes / 2; d > 0; d /= 2) {
            top = max(top, (uint32_t)__shfl_xor(top, d));
            bottom = min(bottom, (uint32_t)__shfl_xor(bottom, d));
        }
    }
    __device__ __forceinline__ uint32_t word() const { return bottom << 16 | top; }
};
__device__ __forceinline__ int row_shift(uint32_t range) { return min(10, 30 - min(30, (int)(range >> 10 & 31))); }
__device__ __forceinline__ bool row_fits(uint32_t range) {
    return (range & 0xffff) < 0x7c00 && ((range >> 16) + 1) << row_shift(range) >= 0x400;
}

// The ranges of a workgroup's rows from m0 on, of stages t0 .. t1 - 1 alone, into LDS.
template <int Rows, int Threads>
__device__ __forceinline__ void find_tile_ranges(const WideArgs& a, uint64_t m0, uint32_t t0, uint32_t t1, uint32_t* ranges) {
    constexpr uint32_t kLanes = Threads / Rows;
    const uint32_t row = threadIdx.x / kLanes;
    const uint16_t* x = a.x + min(m0 + row, a.m - 1) * a.x_stride;
    const uint64_t end = min((uint64_t)t1 * kWideStep, a.depth);
    RowRange range;
#pragma unroll 4
    for (uint64_t c = (uint64_t)t0 * kWideStep + threadIdx.x % kLanes * 8; c < end; c += kLanes * 8)
        range.add(*reinterpret_cast<const u32x4*>(x + c));
    range.join(kLanes);
    if (threadIdx.x % kLanes == 0) ranges[row] = range.word();
    __syncthreads();
}

// A vector of float16 as the sum of two in bfloat16: the leading eight bits of
// each element and the rest.  An infinity or a NaN is whole in the first.
__device__ __forceinline__ void split_half(u32x4 v, u32x4& hi, u32x4& lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t first[2], rest[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t half = v[i] >> 16 * e & 0xffff, size = half & 0x7fff;
            const float f = (float)__builtin_bit_cast(_Float16, (uint16_t)half);
            const uint32_t bits = __float_as_uint(f);
            const float left = f - __uint_as_float(bits & 0xffff0000);
            // a NaN whose payload is all in the lower half must not become an infinity
            first[e] = bits >> 16 | (size > 0x7c00 ? 0x40u : 0u);
            rest[e] = size >= 0x7c00 ? 0u : __float_as_uint(left) >> 16;
        }
        hi[i] = first[0] | first[1] << 16;
        lo[i] = rest[0] | rest[1] << 16;
    }
}

// Keeps products between the reads before and after them.  Matrix instructions
// have no order of their own against loads and barriers: the compiler puts a
// stage's products off past its barrier, and holds all of its fragments till
// then in more registers than there are, or makes them before the reads that
// they are meant to hide.
template <int FM, int FN>
__device__ __forceinline__ void pin(f32x16 (&acc)[FN][FM]) {
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int m = 0; m < FM; ++m) asm volatile("" : "+v"(acc[n][m]));
}

// A wave's accumulators to memory: element 4 q + i of fragment [n][m] is, in lane
// (r, h) of two halves of 32, column n * 32 + 8 q + 4 h + i of row m * 32 + r.
// Stored from there a lane would write 8 bytes of a row of its own, so 32 rows
// by as many columns as are 128 bytes (or as the wave has) go through `turn` (this
// wave's alone) at a time, and eight lanes write a row's 128 bytes.
constexpr uint32_t kTurnBytes = 32 * 128;
template <int FM, int FN, typename T>
__device__ __forceinline__ void store_tile(const f32x16 (&acc)[FN][FM], const OutArgs& o, uint64_t m0, uint64_t j0, T* out,
                                           uint8_t* turn) {
    constexpr int kFragments = FN == 1 ? 1 : 4 / sizeof(T), kCols = kFragments * 32, kChunk = 16 / sizeof(T);
    constexpr uint32_t kLanes = kCols / kChunk, kRows = 64 / kLanes;
    static_assert(FN % kFragments == 0, "");
    const uint32_t lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    out += blockIdx.y * o.split_stride;
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n0 = 0; n0 < FN; n0 += kFragments) {
#pragma unroll
            for (int n = 0; n < kFragments; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    T v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(acc[n0 + n][m][4 * q + i]);
                    const uint32_t col = n * 32 + q * 8 + h * 4;
                    __builtin_memcpy(turn + chunk_at(r, col / kChunk) + col % kChunk * sizeof(T), v, sizeof v);
                }
            wave_sync();
            const uint64_t row0 = m0 + m * 32, col0 = j0 + n0 * 32;
            if (o.vector) {
#pragma unroll
                for (uint32_t i = 0; i < 32 / kRows; ++i) {
                    const uint32_t row = i * kRows + lane / kLanes;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(turn + chunk_at(row, lane % kLanes));
                    const uint64_t col = col0 + lane % kLanes * kChunk;
                    if (row0 + row >= o.m) continue;
                    T* p = out + (row0 + row) * o.stride + col;
                    if (col + kChunk <= o.cols) {
                        *reinterpret_cast<u32x4*>(p) = v;
                    } else {
                        T e[kChunk];
                        __builtin_memcpy(e, &v, sizeof e);
#pragma unroll
                        for (int k = 0; k < kChunk; ++k)
                            if (col + k < o.cols) p[k] = e[k];
                    }
                }
            } else {
                for (uint32_t i = lane; i < 32 * kCols; i += 64) {
                    const uint32_t row = i / kCols, c = i % kCols;
                    T v;
                    __builtin_memcpy(&v, turn + chunk_at(row, c / kChunk) + c % kChunk * sizeof(T), sizeof v);
                    if (row0 + row < o.m && col0 + c < o.cols) out[(row0 + row) * o.stride + col0 + c] = v;
                }
            }
            wave_sync();
        }
}

// Both sides in MX FP4.
struct NarrowArgs {
    const u32x4* x_codes;
    const uint8_t* x_scales;
    const u32x4* w_codes;
    const uint8_t* w_scales;
    uint64_t m, n, blocks, scale_pitch;
    uint32_t steps;
    uint32_t tiles_m, tiles_j;
    OutArgs out_args;
};
int32_t launch_narrow(const NarrowArgs& a, uint32_t tile, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream);
constexpr uint32_t kNarrowStep = 512;  // depth whose scales are loaded together

// At most 32 rows of x in MX FP4 (x_scales set), 16 in other types.
struct SkinnyArgs {
    const void* x;
    const uint8_t* x_scales;
    uint64_t m, n, depth, x_stride;
    uint32_t x_dtype;
    uint32_t vector;  // rows of x start on 16 bytes
    const u32x4* w_codes;
    const uint8_t* w_scales;
    uint64_t blocks, scale_pitch;
    uint32_t groups;  // of 512 of the depth
    void* out;
    uint64_t out_stride;
    uint32_t out_dtype;
};
int32_t launch_skinny(const SkinnyArgs& a, hipStream_t stream);

// half: x is in float16
int32_t launch_wide(const WideArgs& a, bool half, uint32_t tile_m, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream);
int32_t launch_grad(const WideArgs& a, bool half, uint32_t tile_m, uint32_t splits, void* out, uint32_t out_dtype, hipStream_t stream);
// Rows of x and columns of the output a workgroup holds; small tiles may be 64 or
// 32 rows tall (`tile_m`) where x is not in MX FP4.
constexpr uint32_t kLargeTile = 256, kSmallTile = 128;

}  // namespace sllm
