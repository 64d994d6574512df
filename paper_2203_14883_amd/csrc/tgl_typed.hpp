// tgl_typed.hpp -- what the products of rows with their type's weights share:
// arguments, the way from a tile's number to its type and rows, pieces of
// rows and the matrix instructions.
#pragma once

#include "tgl_int8.hpp"

namespace tgl {

using f32x16 = float __attribute__((ext_vector_type(16)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using i16x4 = short __attribute__((ext_vector_type(4)));

struct Groups {
    const int32_t *order;       // or null: rows in their types' order
    const int64_t *offsets;
    int64_t n;
    int32_t num_types;
};

// A number that all lanes have, held once for all.
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(static_cast<uint64_t>(v) >> 32));
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// A stretch of the rows of one type: places [begin, end) of order.
struct Stretch {
    int32_t type;               // num_types for rows of no type
    int32_t count;              // stretches of the type
    int32_t index;              // this one's number among them
    int64_t begin, end;
};

// The places of 64 types from `first` on, a lane each, cut into stretches of
// `rows`: types without rows have `least`, and the rows of no type follow the last
// type where kNone.
template <bool kNone>
__device__ __forceinline__ int32_t stretches_of(const Groups &g, int first, int32_t rows, int32_t least, int64_t &begin, int64_t &end) {
    const int t = first + lane_id();
    begin = end = 0;
    if (t >= g.num_types + (kNone ? 1 : 0)) return 0;
    begin = t == 0 ? 0 : g.offsets[t];
    end = t == g.num_types ? g.n : g.offsets[t + 1];
    begin = begin < 0 ? 0 : begin > g.n ? g.n : begin;
    end = end > g.n ? g.n : end < begin ? begin : end;
    const int32_t count = static_cast<int32_t>((end - begin + rows - 1) / rows);
    return count < least ? least : count;
}

// Stretches in all.  Asked by whole wavefronts, as the next is.
template <bool kNone>
__device__ __forceinline__ uint32_t count_stretches(const Groups &g, int32_t rows, int32_t least) {
    uint32_t all = 0;
    for (int first = 0; first < g.num_types + (kNone ? 1 : 0); first += kWave) {
        int64_t begin, end;
        const uint32_t upto = wave_inclusive_sum(static_cast<uint32_t>(stretches_of<kNone>(g, first, rows, least, begin, end)));
        all += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return all;
}

// Stretch number `at`; false beyond the last.
template <bool kNone>
__device__ __forceinline__ bool find_stretch(const Groups &g, uint32_t at, int32_t rows, int32_t least, Stretch &s) {
    uint32_t before = 0;
    for (int first = 0; first < g.num_types + (kNone ? 1 : 0); first += kWave) {
        int64_t begin, end;
        const int32_t count = stretches_of<kNone>(g, first, rows, least, begin, end);
        const uint32_t upto = before + wave_inclusive_sum(static_cast<uint32_t>(count));
        const uint64_t past = __ballot(at < upto);
        if (past) {
            const int lane = __builtin_ctzll(past);
            s.type = first + lane;
            s.count = __builtin_amdgcn_readlane(count, lane);
            s.index = static_cast<int32_t>(at - (__builtin_amdgcn_readlane(upto, lane) - s.count));
            const int64_t b = uniform(__shfl(begin, lane, kWave)), e = uniform(__shfl(end, lane, kWave));
            s.begin = b + static_cast<int64_t>(s.index) * rows;
            s.end = s.begin + rows < e ? s.begin + rows : e;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return false;
}

// The stretches of a type and, in first, how many there are before them.
__device__ __forceinline__ int32_t stretches_of_type(const Groups &g, int32_t type, int32_t rows, int32_t least, int64_t &first) {
    first = 0;
    for (int t = 0;; t += kWave) {
        int64_t begin, end;
        const int32_t count = stretches_of<false>(g, t, rows, least, begin, end);
        const uint32_t upto = wave_inclusive_sum(static_cast<uint32_t>(count));
        if (type < t + kWave) {
            const int32_t own = __builtin_amdgcn_readlane(count, type - t);
            first += __builtin_amdgcn_readlane(upto, type - t) - own;
            return own;
        }
        first += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
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

}  // namespace tgl
