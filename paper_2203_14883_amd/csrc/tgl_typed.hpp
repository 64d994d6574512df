// tgl_typed.hpp -- what the products of rows with their type's weights share:
// arguments, the way from a tile's number to its type and rows, pieces of
// rows and the matrix instructions.
#pragma once

#include "tgl_int8.hpp"

namespace tgl {

using f32x16 = float __attribute__((ext_vector_type(16)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));

struct Groups {
    const int32_t *order;       // or null: rows in their types' order
    const int64_t *offsets;
    int64_t n;
    int32_t num_types;
};

// A stretch of the rows of one type: places [begin, end) of order.
struct Stretch {
    int32_t type;               // num_types for rows of no type
    int32_t count;              // stretches of the type
    int32_t index;              // this one's number among them
    int64_t begin, end;
};

// Stretch number `at` when every type's rows are cut into stretches of `rows`;
// types without rows have `least` of them, and the rows of no type come last
// where kNone.  False beyond the last.  Asked by whole wavefronts.
template <bool kNone>
__device__ __forceinline__ bool find_stretch(const Groups &g, uint32_t at, int32_t rows, int32_t least, Stretch &s) {
    const int types = g.num_types + (kNone ? 1 : 0);
    uint32_t before = 0;
    for (int first = 0; first < types; first += kWave) {
        const int t = first + lane_id();
        int64_t begin = 0, end = 0;
        int32_t count = 0;
        if (t < types) {
            begin = t == 0 ? 0 : g.offsets[t];
            end = t == g.num_types ? g.n : g.offsets[t + 1];
            begin = begin < 0 ? 0 : begin > g.n ? g.n : begin;
            end = end > g.n ? g.n : end < begin ? begin : end;
            count = static_cast<int32_t>((end - begin + rows - 1) / rows);
            if (count < least) count = least;
        }
        const uint32_t upto = before + wave_inclusive_sum(static_cast<uint32_t>(count));
        const uint64_t past = __ballot(at < upto);
        if (past) {
            const int lane = __builtin_ctzll(past);
            s.type = first + lane;
            s.count = __builtin_amdgcn_readlane(count, lane);
            s.index = static_cast<int32_t>(at - (__builtin_amdgcn_readlane(upto, lane) - s.count));
            const int64_t b = __shfl(begin, lane, kWave), e = __shfl(end, lane, kWave);
            s.begin = b + static_cast<int64_t>(s.index) * rows;
            s.end = s.begin + rows < e ? s.begin + rows : e;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return false;
}

// The row at a place of order, or -1 if there is none.
__device__ __forceinline__ int64_t row_at(const Groups &g, int64_t place, int64_t end) {
    if (place >= end) return -1;
    const int64_t row = g.order ? g.order[place] : place;
    return row >= 0 && row < g.n ? row : -1;
}

// ---- 16 bytes of a row ----

template <class T>
constexpr int kPiece = 16 / static_cast<int>(sizeof(T));

// Elements [c, c + kPiece) of a row of `dim`, zeros beyond and without a row.
template <class T>
__device__ __forceinline__ i32x4 load_piece(const T *row, int c, int dim) {
    using word_t = i32x4 __attribute__((aligned(alignof(T))));
    if (!row || c >= dim) return i32x4{0, 0, 0, 0};
    if (c + kPiece<T> <= dim) return *reinterpret_cast<const word_t *>(row + c);
    Run<T, kPiece<T>> v = {};
#pragma unroll
    for (int i = 0; i < kPiece<T>; i++)
        if (c + i < dim) v.t[i] = row[c + i];
    return __builtin_bit_cast(i32x4, v);
}

// ---- matrix instructions: 16 x 16 outputs of a piece a lane ----
//
// Lane l holds a piece of row l % 16 of each operand.  Which elements of the
// sum's axis it stands for does not matter as long as both operands agree.

template <class T>
__device__ __forceinline__ f32x4 multiply_pieces(const i32x4 &a, const i32x4 &b, f32x4 acc) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; i++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], acc, 0, 0, 0);
        return acc;
    }
}

}  // namespace tgl
