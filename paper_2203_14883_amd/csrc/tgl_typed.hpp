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

// What one lane has, for all.
__device__ __forceinline__ int64_t lane_of(int64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(static_cast<uint64_t>(v) >> 32), lane);
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// A stretch of the rows of one type: places [begin, end) of order.
struct Stretch {
    int32_t type;               // num_types for rows of no type
    int32_t count;              // stretches of the type
    int32_t index;              // this one's number among them
    uint32_t part;              // and among those of types that are cut into several
    int64_t begin, end;
};

// Inclusive sum over the 64 lanes, in registers: these sums stand before every tile's first load.
__device__ __forceinline__ uint32_t lanes_sum(uint32_t v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // within rows of 16: 1, 2, 4, 8 lanes below
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // a row's last to the row above it
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // the lower half's last to the upper half
    return v;
}

// The types of a call, 64 at a time, cut into stretches of `rows` places: types
// without rows have `least`.  Asked by whole wavefronts, whose lanes have a type each.
struct Stretches {
    const Groups &g;
    int32_t rows, least, even;  // even > 0: a type's stretches are alike, in units of `even` places
    int64_t begin, end;         // of the lane's type
    int32_t count;
    uint32_t upto, upto_cut;    // stretches of types up to the lane's, from `first` on; of those that are cut

    __device__ __forceinline__ Stretches(const Groups &g_, int32_t rows_, int32_t least_, int32_t even_)
        : g(g_), rows(rows_), least(least_), even(even_) {}

    __device__ __forceinline__ void take(int first) {
        const int t = first + lane_id();
        begin = end = 0;
        count = 0;
        if (t < g.num_types) {
            begin = t == 0 ? 0 : g.offsets[t];
            end = g.offsets[t + 1];
            begin = begin < 0 ? 0 : begin > g.n ? g.n : begin;
            end = end > g.n ? g.n : end < begin ? begin : end;
            count = static_cast<int32_t>((end - begin + rows - 1) / rows);
            if (count < least) count = least;
        }
        upto = lanes_sum(static_cast<uint32_t>(count));
        if (even > 0) upto_cut = lanes_sum(count > 1 ? static_cast<uint32_t>(count) : 0u);
    }
    // Stretches in all.
    __device__ __forceinline__ uint32_t all() {
        uint32_t sum = 0;
        for (int first = 0; first < g.num_types; first += kWave) {
            take(first);
            sum += __builtin_amdgcn_readlane(upto, kWave - 1);
        }
        return sum;
    }
    // Stretch number `at`; false beyond the last.  After all().
    __device__ __forceinline__ bool find(uint32_t at, Stretch &s) {
        uint32_t before = 0, before_cut = 0;
        for (int first = 0; first < g.num_types; first += kWave) {
            if (g.num_types > kWave) take(first);           // otherwise they are still there
            const uint64_t past = __ballot(at < before + upto);
            if (past) {
                const int lane = __builtin_ctzll(past);
                s.type = first + lane;
                s.count = __builtin_amdgcn_readlane(count, lane);
                s.index = static_cast<int32_t>(at - (before + __builtin_amdgcn_readlane(upto, lane) - s.count));
                const int64_t b = lane_of(begin, lane), e = lane_of(end, lane);
                int32_t each = rows;
                s.part = even > 0 ? before_cut + __builtin_amdgcn_readlane(upto_cut, lane) - s.count + s.index : 0;
                if (even > 0 && s.count > 1) each = static_cast<int32_t>((e - b + s.count - 1) / s.count + even - 1) / even * even;
                s.begin = b + static_cast<int64_t>(s.index) * each;
                s.end = s.begin + each < e ? s.begin + each : e;
                return true;
            }
            before += __builtin_amdgcn_readlane(upto, kWave - 1);
            if (even > 0) before_cut += __builtin_amdgcn_readlane(upto_cut, kWave - 1);
        }
        return false;
    }
    // The number of a type's stretches and, in before, of those of cut types before them.
    __device__ __forceinline__ int32_t of_type(int32_t type, int64_t &before) {
        before = 0;
        for (int first = 0;; first += kWave) {
            take(first);
            if (type < first + kWave) {
                const int32_t own = __builtin_amdgcn_readlane(count, type - first);
                before += __builtin_amdgcn_readlane(upto_cut, type - first) - (own > 1 ? own : 0);
                return own;
            }
            before += __builtin_amdgcn_readlane(upto_cut, kWave - 1);
        }
    }
};

// Where the rows of no type begin.
__device__ __forceinline__ int64_t typed_rows(const Groups &g) {
    const int64_t v = g.offsets[g.num_types];
    return v < 0 ? 0 : v > g.n ? g.n : v;
}

// The row at a place of order, or -1 if there is none.
__device__ __forceinline__ int64_t row_at(const Groups &g, int64_t place, int64_t end) {
    if (place >= end) return -1;
    const int64_t row = g.order ? g.order[place] : place;
    return row >= 0 && row < g.n ? row : -1;
}

// The same at N places, place(0), place(1), ..., of [begin, end), which is not empty: all of them
// on their way at a time.
template <int N, class F>
__device__ __forceinline__ void rows_at(const Groups &g, int64_t end, const F &place, int32_t (&row)[N]) {
    if (g.order) {
#pragma unroll
        for (int i = 0; i < N; i++) row[i] = g.order[place(i) < end ? place(i) : end - 1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) row[i] = static_cast<int32_t>(place(i));
    }
#pragma unroll
    for (int i = 0; i < N; i++)
        if (place(i) >= end || row[i] >= g.n) row[i] = -1;
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
