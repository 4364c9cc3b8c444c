// What the attention kernels share: their arguments, the tiles of keys and values in
// LDS, the way a matrix of scores becomes an operand of the next product.
#pragma once

#include "operators.hpp"
#include "products.hpp"

namespace sllm {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Rows of a tile in LDS are of `D` elements, the head's and zeros after them.  A row is cut
// into chunks of 16 bytes whose order depends on the row, so that 16 rows read in one
// column of chunks, by 16 neighbouring lanes, and four rows read 64 bytes wide are both in
// all 64 banks once.  The place of chunk c ^ d is that of c, exclusive or 16 d.
template <typename T, int D>
struct RowTile {
    static constexpr uint32_t kElements = 16 / sizeof(T), kChunks = D / kElements, kPitch = D * sizeof(T);
    static constexpr uint32_t kLoadRows = 64 / kChunks;  // whose chunks a wave loads at once
    static_assert(kChunks == 8 || kChunks == 16 || kChunks == 32, "");

    static __device__ __forceinline__ uint32_t turn(uint32_t row) {
        return kChunks == 8 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
    }
    static __device__ __forceinline__ uint32_t at(uint32_t row, uint32_t chunk) { return row * kPitch + (chunk ^ turn(row)) * 16; }
};

// `Rows` rows into LDS, by all waves: row r from at(r), zeros where that is null.  Vec:
// rows start on 16 bytes and are whole chunks; loads then go past the registers.
template <typename T, int D, int Rows, int Waves, bool Vec, typename At>
__device__ __forceinline__ void stage_rows(uint8_t* to, uint32_t dim, const At& at) {
    typedef RowTile<T, D> Tile;
    constexpr uint32_t kLoads = Rows / Tile::kLoadRows / Waves;
    static_assert(kLoads * Tile::kLoadRows * Waves == Rows, "");
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const void* const zeros = zero_vector();
#pragma unroll
    for (uint32_t q = 0; q < kLoads; ++q) {
        const uint32_t i = q * Waves + wave, row = i * Tile::kLoadRows + lane / Tile::kChunks;
        const uint32_t e = ((lane % Tile::kChunks) ^ Tile::turn(row)) * Tile::kElements;
        const T* p = at(row);
        if constexpr (Vec) {
            const void* from = p + e;
            load_to_lds(p && e < dim ? from : zeros, to, i * 1024);
        } else {
            T v[Tile::kElements];
#pragma unroll
            for (uint32_t k = 0; k < Tile::kElements; ++k) v[k] = p && e + k < dim ? p[e + k] : (T)0.0f;
            lds_write(to, i * 1024 + lane * 16, __builtin_bit_cast(u32x4, v));
        }
    }
}

// The same from rows that are whole and whose places repeat: row r + kRun n of a tile is n
// times `step` bytes behind row r.  A lane then needs one place of its own, or where its
// chunk changes from load to load two.
template <typename T, int D, int Rows, int Waves>
struct LaneOffsets {
    typedef RowTile<T, D> Tile;
    static constexpr uint32_t kLoads = Rows / Tile::kLoadRows / Waves, kRun = Waves * Tile::kLoadRows < 16 ? 16 : Waves * Tile::kLoadRows;
    static constexpr uint32_t kPlaces = kRun / (Waves * Tile::kLoadRows);
    uint32_t bytes[kPlaces];
    uint64_t step;

    template <typename At>  // element offset of row r, below kRun
    __device__ __forceinline__ void set(uint64_t step_elements, const At& at) {
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        step = step_elements * sizeof(T);
#pragma unroll
        for (uint32_t q = 0; q < kPlaces; ++q) {
            const uint32_t row = (q * Waves + wave) * Tile::kLoadRows + lane / Tile::kChunks;
            bytes[q] = (uint32_t)(at(row) + ((lane % Tile::kChunks) ^ Tile::turn(row)) * Tile::kElements) * (uint32_t)sizeof(T);
        }
    }
    __device__ __forceinline__ void stage(uint8_t* to, const T* base) const {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (uint32_t q = 0; q < kLoads; ++q)
            load_to_lds(reinterpret_cast<const uint8_t*>(base) + q / kPlaces * step + bytes[q % kPlaces], to, (q * Waves + wave) * 1024);
    }
};

// Eight elements of a lane: an operand of 16 of the depth by 32 rows or columns, of which
// lane (r, h) has row r and depths 8 h to 8 h + 7.
template <typename T>
struct Operand8 {
    u32x4 v;
};
template <>
struct Operand8<float> {
    f32x8 v;
};

template <typename T>
__device__ __forceinline__ f32x16 multiply(const Operand8<T>& a, const Operand8<T>& b, f32x16 acc) {
    if constexpr (__is_same(T, float)) {
        // two depths an instruction, one a half wave: which does not matter if both sides agree
#pragma unroll
        for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], acc, 0, 0, 0);
        return acc;
    } else {
        return product<T>(a.v, b.v, acc);
    }
}

// Of rows row0 to row0 + 31 of a tile, step s of 16 of their elements.
template <typename T, int D>
__device__ __forceinline__ Operand8<T> read_rows(const uint8_t* tile, uint32_t from, int row0, int s) {
    Operand8<T> o;
    if constexpr (__is_same(T, float)) {
        const f32x4 a = lds_read<f32x4>(tile, (from ^ s * 64) + row0 * RowTile<T, D>::kPitch);
        const f32x4 b = lds_read<f32x4>(tile, (from ^ (s * 64 + 16)) + row0 * RowTile<T, D>::kPitch);
        o.v = f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    } else {
        o.v = lds_read<u32x4>(tile, (from ^ s * 32) + row0 * RowTile<T, D>::kPitch);
    }
    return o;
}
// The `from` of a lane.
template <typename T, int D>
__device__ __forceinline__ uint32_t rows_from(uint32_t lane) {
    return opaque(RowTile<T, D>::at(lane & 31, (lane >> 5) * (sizeof(T) / 2)));
}

// Scores come out of a product in registers: of a matrix of 32 rows, lane (c, h) has
// column c and rows 8 (i / 4) + 4 h + i % 4.  Eight of them, 16 rows in the two halves,
// are an operand over those rows as they are, if the other side takes the rows in that
// order: the rows of a tile, element by element, in lane (element, h).
template <typename T, int D>
__device__ __forceinline__ Operand8<T> read_columns(const uint8_t* tile, uint32_t from, int row0, int column0) {
    Operand8<T> o;
    if constexpr (__is_same(T, float)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // rows row0 + 8 (j / 4) + 4 h + j % 4: their turn is (j % 4) << 2 | (2 (j / 4) + h)
            const uint32_t turn = RowTile<T, D>::kChunks == 8 ? (j >> 1 & 1) << 6 | (j >> 2) << 5 : (j & 3) << 6 | (j >> 2) << 5;
            o.v[j] = lds_read<float>(tile, (from ^ turn ^ column0 * 4) + (row0 + 8 * (j / 4) + j % 4) * RowTile<T, D>::kPitch);
        }
    } else {
        // 16 lanes read four rows of 16 elements and get a column of four each
        typedef __attribute__((address_space(3))) i16x4 Lds;
        u32x2 part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = (from ^ column0 * 2 ^ u * 32) + (row0 + 8 * u) * RowTile<T, D>::kPitch;
            part[u] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)((lds_u8*)tile + at)));
        }
        o.v = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
    }
    return o;
}
template <typename T, int D>
__device__ __forceinline__ uint32_t columns_from(uint32_t lane) {
    typedef RowTile<T, D> Tile;
    if constexpr (__is_same(T, float)) {
        const uint32_t row = 4 * (lane >> 5), c = lane & 31;
        return opaque(Tile::at(row, c / 4) + c % 4 * 4);
    } else {
        const uint32_t row = 4 * (lane >> 5) + (lane >> 2 & 3), c = (lane >> 4 & 1) * 16 + (lane & 3) * 4;
        return opaque(Tile::at(row, c / 8) + c % 8 * 2);
    }
}

// Registers 8 t to 8 t + 7 as an operand, rounded to nearest even.
template <typename T>
__device__ __forceinline__ Operand8<T> as_operand(const f32x16& x, int t) {
    Operand8<T> o;
    if constexpr (__is_same(T, float)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = x[8 * t + j];
    } else {
        typedef T T2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            o.v[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[8 * t + 2 * j], x[8 * t + 2 * j + 1]}, T2));
    }
    return o;
}

// What rounding to an operand has left of them.
template <typename T>
__device__ __forceinline__ f32x16 rounded_off(const f32x16& x, const Operand8<T> (&o)[2]) {
    f32x16 rest;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        T v[8];
        __builtin_memcpy(v, &o[t].v, sizeof v);
#pragma unroll
        for (int j = 0; j < 8; ++j) rest[8 * t + j] = x[8 * t + j] - to_f32(v[j]);
    }
    return rest;
}

// Eight elements of a row in memory from element e, zeros past its end.
template <typename T, bool Vec>
__device__ __forceinline__ Operand8<T> load8(const T* row, uint32_t e, uint32_t dim) {
    T v[8];
    if constexpr (Vec) {
        constexpr uint32_t n = 16 / sizeof(T);
#pragma unroll
        for (uint32_t i = 0; i < 8 / n; ++i) {
            u32x4 raw = {0, 0, 0, 0};
            if (e + i * n < dim) raw = *reinterpret_cast<const u32x4*>(row + e + i * n);
            __builtin_memcpy(v + i * n, &raw, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e + i < dim ? row[e + i] : (T)0.0f;
    }
    Operand8<T> o;
    __builtin_memcpy(&o.v, v, sizeof v);
    return o;
}

// A lane's and that of the same column in the other half wave.
__device__ __forceinline__ f32x2 both_halves(float x) {
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}

// Products with rows of which some columns must see nothing: what is not a number there
// would come through a weight of zero.  Such elements are taken out of the operand, and at
// the end added, as they are, to the columns that see their row.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t word) {  // halves that are not, as all ones
    constexpr uint32_t kExponent = __is_same(T, _Float16) ? 0x7c00 : 0x7f80;
    return ((word & kExponent) == kExponent ? 0xffffu : 0u) | ((word >> 16 & kExponent) == kExponent ? 0xffff0000u : 0u);
}
template <typename T>
__device__ __forceinline__ void take_out(Operand8<T>& o) {
    if constexpr (__is_same(T, float)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            o.v[i] = (__float_as_uint(o.v[i]) & 0x7f800000) == 0x7f800000 ? 0.0f : o.v[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o.v[i] &= ~not_finite<T>(o.v[i]);
        }
    }
}

// Whether any of `Rows` rows at the start of a tile has an element that is not finite: a step
// of the exponent carries into the sign where it is all ones.
template <typename T, int D, int Rows>
__device__ __forceinline__ bool any_not_finite(const uint8_t* tile) {
    constexpr uint32_t kMask = __is_same(T, float) ? 0x7f800000 : __is_same(T, _Float16) ? 0x7c007c00 : 0x7f807f80;
    constexpr uint32_t kStep = __is_same(T, float) ? 0x00800000 : __is_same(T, _Float16) ? 0x04000400 : 0x00800080;
    uint32_t from = (threadIdx.x & 63) * 16, any = 0;
    asm volatile("" : "+v"(from));  // not to be found out before this is reached
#pragma unroll
    for (uint32_t i = 0; i < Rows * RowTile<T, D>::kPitch / 1024; ++i) {
        const u32x4 v = lds_read<u32x4>(tile, i * 1024 + from);
#pragma unroll
        for (int j = 0; j < 4; ++j) any |= (v[j] & kMask) + kStep;
    }
    return __any((any & (__is_same(T, float) ? 0x80000000 : 0x80008000)) != 0);
}

// acc with what was taken out: the elements of a row in memory that are not finite, where
// the lane's column sees it.  To be called for all rows: one that has been added already
// changes nothing the second time.
template <typename T, int D>
__device__ __forceinline__ void put_back(f32x16 (&acc)[D / 32], const T* row, uint32_t dim, bool seen) {
    const uint32_t h = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t e = 32 * d + 8 * (i / 4) + 4 * h + i % 4;
            if (e >= dim) continue;
            const float f = to_f32(row[e]);
            if (seen && !(__builtin_fabsf(f) < __builtin_inff())) acc[d][i] += f;
        }
}

// Keeps what is before it before what is after it.  Fragments are read in runs, a run ahead
// of the products that take them: left alone the compiler reads each just before its own.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// Rows row0 to row0 + 31 of a tile, as operands.
template <typename T, int D>
struct RowFragments {
    Operand8<T> f[D / 16];

    __device__ __forceinline__ void read(const uint8_t* tile, uint32_t from, int row0) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) f[s] = read_rows<T, D>(tile, from, row0, s);
    }
    // their products with the lane's columns
    __device__ __forceinline__ f32x16 times(const Operand8<T> (&columns)[D / 16]) const {
        f32x16 acc = {};
#pragma unroll
        for (int s = 0; s < D / 16; ++s) acc = multiply(f[s], columns[s], acc);
        return acc;
    }
};

// Elements 32 d to 32 d + 31 of `Rows` rows, likewise, for acc += the sum over the rows of
// those times the weight of the lane's column, w[t] being the operand of rows 16 t on.
template <typename T, int D, int Rows>
struct ColumnFragments {
    Operand8<T> f[Rows / 16];

    __device__ __forceinline__ void read(const uint8_t* tile, uint32_t from, int row0, int d) {
#pragma unroll
        for (int t = 0; t < Rows / 16; ++t) f[t] = read_columns<T, D>(tile, from, row0 + 16 * t, 32 * d);
    }
    __device__ __forceinline__ void add(f32x16& acc, const Operand8<T> (&w)[Rows / 16]) const {
#pragma unroll
        for (int t = 0; t < Rows / 16; ++t) acc = multiply(f[t], w[t], acc);
    }
    // those that are not finite becoming zeros
    __device__ __forceinline__ void take_out() {
#pragma unroll
        for (int t = 0; t < Rows / 16; ++t) sllm::take_out(f[t]);
    }
};

// All of them; the first are read already.  bad: there is something to take out.
template <typename T, int D, int Rows>
__device__ __forceinline__ void add_weighted(f32x16 (&acc)[D / 32], ColumnFragments<T, D, Rows>& first, const uint8_t* tile, uint32_t from,
                                             int row0, const Operand8<T> (&w)[Rows / 16], bool bad) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        ColumnFragments<T, D, Rows> next;
        if (d + 1 < D / 32) next.read(tile, from, row0, d + 1);
        if (bad) first.take_out();
        first.add(acc[d], w);
        phase();
        if (d + 1 < D / 32) first = next;
    }
}

// ---------------------------------------------------------------------------
// Softmax
// ---------------------------------------------------------------------------

// What a row's weights are taken against: of a score s, 2^(scale (s - less) - scaled), which
// is 2^kUp for the row's largest so far, or up to 2^kSlack times that.  float16 has the least
// of such weights as normal numbers.  Scores so large that a rounded `scaled` would be off by
// more than 2^-8 have their own largest taken away first.
template <typename T>
struct Reference {
    static constexpr float kUp = __is_same(T, _Float16) ? 7.0f : 0.0f, kSlack = 8.0f, kFar = 0x1p16f;
    float most = -__builtin_inff(), less = 0, scaled = 0;

    // The row's largest is now `next`: what is made of the sums so far.
    __device__ __forceinline__ float raise(float next, float scale) {
        const bool none = next == -__builtin_inff();
        const float next_less = sizeof(T) == 2 && !none && __builtin_fabsf(next * scale) > kFar ? next : 0.0f;
        const float next_scaled = none ? -kUp : __builtin_fmaf(next - next_less, scale, -kUp);
        const float down = sizeof(T) == 4 ? (most - next) * scale : __builtin_fmaf(less - next_less, scale, scaled) - next_scaled;
        const float f = __builtin_amdgcn_exp2f(most == -__builtin_inff() ? 0.0f : down);
        most = next, less = next_less, scaled = next_scaled;
        return f;
    }
    __device__ __forceinline__ float weight(float s, float scale, float finite) const {
        // (the difference first is exact near the largest score, which 16 bits do not tell)
        return __builtin_amdgcn_exp2f(sizeof(T) == 4 ? (s - finite) * scale : __builtin_fmaf(s, scale, -scaled));
    }
    __device__ __forceinline__ float finite() const { return most == -__builtin_inff() ? 0.0f : most; }
    // What makes sums of weights those against scale * most - kUp, without its rounding.
    __device__ __forceinline__ float exact(float scale) const {
        return sizeof(T) == 4 || most == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(kUp - __builtin_fmaf(most - less, scale, -scaled));
    }
    // log2 of the sum of 2^(scale s), of that of weights
    __device__ __forceinline__ float log_sum(float sum, float scale) const {
        const float l = __builtin_amdgcn_logf(sum);
        return sizeof(T) == 4 ? __builtin_fmaf(most, scale, l) : __builtin_fmaf(less, scale, scaled + l);
    }
};

// ---------------------------------------------------------------------------
// Sequences
// ---------------------------------------------------------------------------

__device__ __forceinline__ int64_t read_id(const void* ids, bool wide, uint64_t i) {
    return wide ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}

// How many tokens a sequence has had, -1 where it takes no part.  Past 2^62 positions would
// leave 64 bits.
__device__ __forceinline__ int64_t read_length(const AttentionArgs& a, uint32_t s) {
    const int64_t n = read_id(a.lengths, a.wide_lengths, s);
    return n > 1ll << 62 ? -1 : n;
}

// A piece of a sequence: tokens first .. first + n - 1 of the packed rows, and which
// piece of it.  None: n = 0, then `piece` counts those past the last one, of `spare`, and
// rows before `first` and from `past_end` on belong to no sequence.
struct Piece {
    uint32_t sequence, first, n, piece, spare, past_end;
};

// Piece `index` of all sequences, each cut into ceil(tokens * rows / size).  Offsets are
// taken as far as they do not go back and lie within the tokens, so that no two sequences
// share a row whatever they hold.  A wave reads 64 sequences at a time.
__device__ __forceinline__ Piece find_piece(const void* offsets, bool wide, uint32_t sequences, uint32_t tokens, uint32_t rows,
                                            uint32_t size, uint32_t index, uint32_t pieces) {
    const auto cut = [&](uint32_t n) { return (uint32_t)(((uint64_t)n * rows + size - 1) / size); };
    if (!offsets) {
        const uint32_t all = cut(tokens);
        if (index < all) return {0, 0, tokens, index, 0, tokens};
        return {0, 0, 0, index - all, pieces - all, tokens};
    }
    const uint32_t lane = threadIdx.x & 63;
    uint32_t before = 0, start = 0, first_row = 0;  // pieces so far, where the last sequence ended
    for (uint32_t s0 = 0; s0 < sequences; s0 += 64) {
        // the ends of sequences s0 .., at least each one's start and the ends before
        const uint32_t s = s0 + lane;
        const auto clamp = [&](int64_t v) { return (uint32_t)min(max(v, (int64_t)0), (int64_t)tokens); };
        if (s0 == 0) first_row = start = __builtin_amdgcn_readfirstlane(clamp(read_id(offsets, wide, 0)));
        uint32_t end = s < sequences ? clamp(read_id(offsets, wide, s + 1)) : 0;
        end = max(end, start);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = __shfl_up(end, d);
            if (lane >= (uint32_t)d) end = max(end, v);
        }
        uint32_t from = __shfl_up(end, 1);
        if (lane == 0) from = start;
        const uint32_t mine = s < sequences ? cut(end - from) : 0;
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = __shfl_up(upto, d);
            if (lane >= (uint32_t)d) upto += v;
        }
        const uint64_t found = __ballot(before + upto > index);
        if (found) {
            const int at = __builtin_ctzll(found);
            const uint32_t f = __builtin_amdgcn_readlane(from, at), e = __builtin_amdgcn_readlane(end, at);
            return {s0 + at, f, e - f, index - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at)), 0, 0};
        }
        before += __builtin_amdgcn_readlane(upto, 63);
        start = __builtin_amdgcn_readlane(end, 63);
    }
    return {0, first_row, 0, index - before, pieces - before, start};
}

// The tile of a workgroup: neighbouring ones of a head on one XCD, whose L2 then holds its keys.
__device__ __forceinline__ uint32_t xcd_index() {
    const uint32_t xcd = blockIdx.x % 8, q = gridDim.x / 8, rest = gridDim.x % 8;
    return xcd * q + min(xcd, rest) + blockIdx.x / 8;
}

// Zeros into the share of a workgroup without a piece: rows `head0` .. + heads - 1 of
// tokens that belong to no sequence.
template <typename T>
__device__ __forceinline__ void clear_spare(const Piece& p, uint32_t tokens, T* out, uint64_t token_stride, uint64_t head_stride,
                                            uint32_t head0, uint32_t heads, uint32_t dim) {
    const uint32_t n = tokens - (p.past_end - p.first);
    for (uint32_t t = p.piece; t < n; t += p.spare) {
        const uint64_t token = t < p.first ? t : t - p.first + p.past_end;
        for (uint32_t i = threadIdx.x; i < heads * dim; i += blockDim.x)
            out[token * token_stride + (head0 + i / dim) * head_stride + i % dim] = (T)0.0f;
    }
}

// A lane's column of (elements x columns) sums times f, to a row in memory.
template <typename T, int D, bool Vec>
__device__ __forceinline__ void store_column(const f32x16 (&acc)[D / 32], float f, T* row, uint32_t dim) {
    const uint32_t h = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t e = 32 * d + 8 * g + 4 * h;
            T v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(acc[d][4 * g + i] * f);
            if (Vec) {
                if (e < dim) __builtin_memcpy(__builtin_assume_aligned(row + e, 4 * sizeof(T)), v, sizeof v);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e + i < dim) row[e + i] = v[i];
            }
        }
}

// Where sequence s starts and how many tokens it has, as find_piece takes the offsets.
__device__ __forceinline__ void find_sequence(const void* offsets, bool wide, uint32_t s, uint32_t tokens, uint32_t& first, uint32_t& n) {
    first = 0, n = tokens;
    if (!offsets) return;
    const auto clamp = [&](int64_t v) { return (uint32_t)min(max(v, (int64_t)0), (int64_t)tokens); };
    uint32_t most = 0;
    for (uint32_t i = threadIdx.x & 63; i <= s; i += 64) most = max(most, clamp(read_id(offsets, wide, i)));
#pragma unroll
    for (int d = 32; d > 0; d /= 2) most = max(most, (uint32_t)__shfl_xor(most, d));
    first = __builtin_amdgcn_readfirstlane(most);
    n = __builtin_amdgcn_readfirstlane(max(first, clamp(read_id(offsets, wide, s + 1)))) - first;
}

// The keys that the queries at positions i0 to i1 of a sequence see: the first `sinks`
// positions, those not in the window among them, then lo to i1.  Key c of that list is at
// distance c - sinks from lo; positions count from lo, in 32 bits.
struct KeyList {
    int32_t sinks, total;       // keys before lo, all keys
    int32_t early, window;      // positions from lo on below this are sinks too
    int64_t lo;

    __device__ __forceinline__ KeyList(int64_t i0, int64_t i1, int32_t window, int32_t all_sinks) : window(window) {
        lo = max((int64_t)0, i0 - window + 1);
        sinks = (int32_t)min((int64_t)all_sinks, lo);
        early = (int32_t)max((int64_t)0, all_sinks - lo);
        total = sinks + (int32_t)(i1 - lo + 1);
    }
    // What the query at lo + q sees: up to its own key, all but those from the last sink to
    // the window.
    struct Sight {
        int32_t last, hidden;
        uint32_t n_hidden;

        __device__ __forceinline__ bool sees(int32_t c) const { return (c <= last) & ((uint32_t)(c - hidden) >= n_hidden); }
        // the same, not to be found out before this is reached
        __device__ __forceinline__ Sight here() const {
            Sight s = *this;
            asm volatile("" : "+v"(s.last), "+v"(s.hidden), "+v"(s.n_hidden));
            return s;
        }
    };
    __device__ __forceinline__ Sight sight(int32_t q) const {
        const int32_t hidden = sinks + early;
        return {min(q + sinks, total - 1), hidden, (uint32_t)max(0, q + sinks - window + 1 - hidden)};
    }
    // whether all queries lo + q0 .. lo + q1 see keys c0 .. c1, and whether none sees any
    __device__ __forceinline__ bool all(int32_t q0, int32_t q1, int32_t c0, int32_t c1) const {
        return c1 < total && c1 - sinks <= q0 && (c1 - sinks < early || q1 - (c0 - sinks) < window);
    }
    __device__ __forceinline__ bool none(int32_t q0, int32_t q1, int32_t c0, int32_t c1) const {
        return c0 - sinks > q1 || (c0 - sinks >= early && q0 - (c1 - sinks) >= window);
    }
};

}  // namespace sllm
