// tgl_typed_tile.hpp -- a tile of a matrix product on the matrix units: BM x BN
// outputs of a workgroup, whose operands come through LDS in steps of SB bytes
// of the sum's axis.
//
// A side is what one operand brings to a step: B rows of the tile's edge times
// SB bytes of the sum's axis.  It lies in LDS as the memory has it, so that
// loads go straight there, 16 bytes a lane:
//   along   the sum's axis is the one that memory runs along: B rows of SB bytes,
//           and a lane reads a piece of 16 bytes of one row;
//   across  the sum's axis goes from row to row of memory: a row of LDS holds
//           the B elements of one place of the sum's axis, and the reads turn
//           them (bfloat16: the transposing read of LDS; float32: a lane takes
//           four columns, and so a column of four tiles).
// Pieces are permuted within their rows (an exclusive or with bits of the row),
// so that what a read touches lies in different banks.
#pragma once

#include "tgl_typed.hpp"

namespace tgl {

template <class T, int SB>
constexpr int kStep = SB / static_cast<int>(sizeof(T));     // of the sum's axis

using lds_t = __attribute__((address_space(3))) void;

// Where lanes read what is beyond the sum's axis.
static __device__ const i32x4 kZeros = {0, 0, 0, 0};

// 16 bytes a lane from memory straight to LDS, one lane's after another's.  The
// instruction itself, which has no result in registers: for the builtin the
// compiler waits, before reads of any buffer that it cannot tell apart, until all loads
// are done, and with that nothing is on its way any more.  What has to be waited for is in
// meet().  m0, the place in LDS, is an operand that the compiler fills, so that it knows what is there; an
// instruction has to lie between.
__device__ __forceinline__ uint32_t lds_place(const int8_t *to) {
    return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_t *)to)));
}
template <class T>
__device__ __forceinline__ void to_lds(const T *from, int8_t *to) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(lds_place(to)));
}
// The same from one place for all lanes and a number of bytes for each.
template <class T>
__device__ __forceinline__ void to_lds(const T *from, uint32_t bytes, int8_t *to) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(bytes), "s"(from), "{m0}"(lds_place(to)));
}

// Whether a lane's pieces are four columns of one place of the sum's axis
// each (of four tiles), and not four places of one column.
template <class T, bool kAcross, int N>
constexpr bool kQuads = sizeof(T) == 4 && kAcross && N % 4 == 0;

// ---- sides ----
//
// Each wavefront brings kFetch times 1024 bytes of a side.  kDirect: row starts
// and strides are multiples of 16 bytes and so is the sum's axis, or the edge's
// length where it is the one that memory runs along; memory goes straight to LDS.
// Otherwise it goes through registers: fetch() a step ahead, store() after.

// `along`: rows[f] are the lane's rows of the tile's edge.
template <class T, int B, int NW, int SB, bool kDirect>
struct Along {
    static constexpr int kPieces = SB / 16, kRows = kWave / kPieces, kFetch = B / kRows / NW;
    static_assert(B % (kRows * NW) == 0, "the wavefronts fetch as much each");
    const T *row[kFetch];       // kDirect: at the lane's piece
    i32x4 held[kDirect ? 1 : kFetch];
    int length;                 // of the sum's axis

    static __device__ __forceinline__ int swizzle(int r) { return (r >> 1) & (kPieces - 1); }
    static __device__ __forceinline__ int edge(int wave, int f) { return (wave * kFetch + f) * kRows + lane_id() / kPieces; }
    static __device__ __forceinline__ int column(int wave, int f) {
        return ((lane_id() % kPieces) ^ swizzle(edge(wave, f))) * kPiece<T>;
    }

    // A row that is not there may be any row: what comes of it is not stored.
    __device__ __forceinline__ void set(int wave, int f, const T *p) { row[f] = kDirect ? p + column(wave, f) : p; }

    __device__ __forceinline__ void fetch(int wave, int step, int8_t *buf) {
        const int k = step * kStep<T, SB>;
        const bool whole = k + kStep<T, SB> <= length;
#pragma unroll
        for (int f = 0; f < kFetch; f++) {
            if constexpr (kDirect) {
                const T *p = row[f] + k;
                if (!whole && k + column(wave, f) >= length) p = reinterpret_cast<const T *>(&kZeros);
                to_lds(p, buf + (wave * kFetch + f) * 1024);
            } else {
                held[f] = load_piece(row[f], k + column(wave, f), length);
            }
        }
    }
    __device__ __forceinline__ void store(int wave, int8_t *buf) {
        if constexpr (!kDirect)
#pragma unroll
            for (int f = 0; f < kFetch; f++) *reinterpret_cast<i32x4 *>(buf + (wave * kFetch + f) * 1024 + lane_id() * 16) = held[f];
    }
    // The lane's pieces of `N` tiles of 16 rows from `first` on, of 64 bytes h of a step.
    template <int N>
    static __device__ __forceinline__ void read(const int8_t *buf, int side, int first, int h, i32x4 (&v)[N]) {
        const int r = first + (lane_id() & 15);
        const int at = (side + r * SB + (((4 * h + (lane_id() >> 4)) ^ swizzle(r)) * 16));
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = *reinterpret_cast<const i32x4 *>(buf + (at + i * 16 * SB));
    }
};

// What both kinds of `across` share: where a lane's bytes go and come from.
template <class T, int B, int NW, int SB>
struct AcrossLayout {
    static constexpr int kPieces = B * static_cast<int>(sizeof(T)) / 16;      // of a row of LDS
    static constexpr int kRows = kWave / kPieces;                             // of a fetch
    static constexpr int kFetch = kStep<T, SB> / kRows / NW;
    static_assert(kPieces <= kWave && kStep<T, SB> % (kRows * NW) == 0, "the wavefronts fetch as much each");

    static __device__ __forceinline__ int swizzle(int k) {
        if constexpr (sizeof(T) == 4) return k & 12;
        return ((k & 3) << 1) | (kPieces >= 16 ? k & 8 : 0);
    }
    // The lane's place of the sum's axis in a step, and its columns of the edge.
    static __device__ __forceinline__ int place(int wave, int f) { return (wave * kFetch + f) * kRows + lane_id() / kPieces; }
    static __device__ __forceinline__ int column(int wave, int f) {
        return ((lane_id() % kPieces) ^ swizzle(place(wave, f))) * kPiece<T>;
    }

    template <int N>
    static __device__ __forceinline__ void read(const int8_t *buf, int side, int first, int h, i32x4 (&v)[N]) {
        const int i16 = lane_id() & 15, g = lane_id() >> 4;
        if constexpr (sizeof(T) == 2) {
            using words_t = __attribute__((address_space(3))) i16x4;
            const int k = 8 * g + (i16 >> 2);           // + 32 h + 4 q, which the swizzle does not see
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int c = first + 16 * i + 4 * (i16 & 3);
                const int at = (side + (32 * h + k) * (kPieces * 16) + (((c >> 3) ^ swizzle(k)) * 16) + (c & 4) * 2);
                const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((words_t *)(buf + at));
                const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((words_t *)(buf + (at + 4 * kPieces * 16)));
                v[i] = __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        } else if constexpr (kQuads<T, true, N>) {
            // v[4 t + i]: place i of the lane's four, a column of each of tiles 4 t to 4 t + 3
#pragma unroll
            for (int t = 0; t < N / 4; t++) {
                const int at = (side + (16 * h + 4 * g) * (kPieces * 16) + (((first / 4 + 16 * t + i16) ^ (4 * g)) * 16));
#pragma unroll
                for (int i = 0; i < 4; i++) v[4 * t + i] = *reinterpret_cast<const i32x4 *>(buf + (at + i * kPieces * 16));
            }
        } else {
#pragma unroll
            for (int t = 0; t < N; t++) {
                const int c = first + 16 * t + i16;
                const int at = (side + (16 * h + 4 * g) * (kPieces * 16) + (((c >> 2) ^ (4 * g)) * 16) + (c & 3) * 4);
#pragma unroll
                for (int i = 0; i < 4; i++) v[t][i] = *reinterpret_cast<const int *>(buf + (at + i * kPieces * 16));
            }
        }
    }
};

// `across` with rows of memory one after another: a type's weights.
template <class T, int B, int NW, int SB, bool kDirect>
struct Across : AcrossLayout<T, B, NW, SB> {
    using L = AcrossLayout<T, B, NW, SB>;
    using L::kFetch;
    i32x4 held[kDirect ? 1 : kFetch];
    const T *base;
    int64_t stride;
    int length, first, edge;    // of the sum's axis; the tile's first column; columns in all

    __device__ __forceinline__ void set(int wave, const T *base_, int64_t stride_, int length_, int first_, int edge_) {
        base = base_ + wave * (kFetch * L::kRows) * stride_;
        stride = stride_;
        length = length_;
        first = first_;
        edge = edge_;
    }
    __device__ __forceinline__ void fetch(int wave, int step, int8_t *buf) {
        const int k = step * kStep<T, SB>;
        const bool whole = k + kStep<T, SB> <= length;
#pragma unroll
        for (int f = 0; f < kFetch; f++) {
            const int c = first + L::column(wave, f);
            if constexpr (kDirect) {
                // a wavefront's rows begin at one place; the lane's is not far from there
                const T *p = base + (k + f * L::kRows) * stride;
                const uint32_t at = lane_id() / L::kPieces * static_cast<uint32_t>(stride) + (c < edge ? c : 0);
                int8_t *to = buf + (wave * kFetch + f) * 1024;
                if (whole) to_lds(p, at * static_cast<uint32_t>(sizeof(T)), to);
                else to_lds(k + L::place(wave, f) < length ? p + at : reinterpret_cast<const T *>(&kZeros), to);
            } else {
                const bool there = whole || k + L::place(wave, f) < length;
                held[f] = load_piece(there ? base + (k + f * L::kRows + lane_id() / L::kPieces) * stride : nullptr, c, edge);
            }
        }
    }
    __device__ __forceinline__ void store(int wave, int8_t *buf) {
        if constexpr (!kDirect)
#pragma unroll
            for (int f = 0; f < kFetch; f++) *reinterpret_cast<i32x4 *>(buf + (wave * kFetch + f) * 1024 + lane_id() * 16) = held[f];
    }
};

// `across` with rows of memory that places of order name.
template <class T, int B, int NW, int SB, bool kDirect>
struct Gathered : AcrossLayout<T, B, NW, SB> {
    using L = AcrossLayout<T, B, NW, SB>;
    using L::kFetch;
    i32x4 held[kDirect ? 1 : kFetch];
    const T *base;
    int64_t stride;
    int first, edge;

    __device__ __forceinline__ void set(const T *base_, int64_t stride_, int first_, int edge_) {
        base = base_;
        stride = stride_;
        first = first_;
        edge = edge_;
    }
    // places: the step's rows, of which there are none where the number is negative.
    template <class Places>
    __device__ __forceinline__ void fetch(int wave, const Places &places, int8_t *buf) {
        unrolled<kFetch>([&](auto F) {
            constexpr int f = decltype(F)::value;
            const int32_t id = places.template row<L::kRows, f * L::kRows>();
            const int c = first + L::column(wave, f);
            if constexpr (kDirect) {
                // opaque, or base + column of every load would be kept over the steps, in twice the registers: in tiles of 256
                // 10 of them were spilled then (16,384 x 4096 x 4096 of 8 types 1.0 ms, 0.65 without)
                uint32_t column = c < edge ? c : 0;
                asm volatile("" : "+v"(column));
                to_lds(id < 0 ? reinterpret_cast<const T *>(&kZeros) : base + id * stride + column, buf + (wave * kFetch + f) * 1024);
            } else {
                held[f] = load_piece(id < 0 ? nullptr : base + id * stride, c, edge);
            }
        });
    }
    __device__ __forceinline__ void store(int wave, int8_t *buf) {
        if constexpr (!kDirect)
#pragma unroll
            for (int f = 0; f < kFetch; f++) *reinterpret_cast<i32x4 *>(buf + (wave * kFetch + f) * 1024 + lane_id() * 16) = held[f];
    }
};

// The rows of a wavefront's OWN places of a step, a lane each, from order a step
// earlier: looked at only when they are used, since that waits for every load before them.
template <int OWN>
struct Places {
    const int32_t *order;
    int64_t begin;
    int32_t n, places;          // rows of the call; places of the stretch
    int32_t next;               // the lane's place of the next step
    int32_t id, later;          // this step's row, -1 if there is none; the next one's

    __device__ __forceinline__ Places(const Groups &g, int64_t begin_, int64_t end, int32_t first) : order(g.order), begin(begin_) {
        n = static_cast<int32_t>(g.n);
        places = static_cast<int32_t>(end - begin);
        next = first + lane_id() % OWN;
        later = 0;
        load();
    }
    __device__ __forceinline__ void load() {
        if (order) later = order[begin + (next < places ? next : places - 1)];
    }
    // On to a step, of which there is one after every `by` places.
    __device__ __forceinline__ void advance(int32_t by) {
        id = order ? later : static_cast<int32_t>(begin) + next;
        if (next >= places || id >= n) id = -1;
        next += by;
    }
    // The lane's of N places from the wavefront's number FROM on.
    template <int N, int FROM>
    __device__ __forceinline__ int32_t row() const {
        return __shfl(id, FROM + lane_id() / (kWave / N), kWave);
    }
};

// ---- products of what was read ----
//
// float32: what a lane has of tile t at place k of its four.
template <class T, bool kAcross, int N>
__device__ __forceinline__ float element(const i32x4 (&v)[N], int t, int k) {
    if constexpr (kQuads<T, kAcross, N>) return __builtin_bit_cast(f32x4, v[t / 4 * 4 + k])[t % 4];
    else return __builtin_bit_cast(f32x4, v[t])[k];
}

// acc[first + i][j] += x[i] w[j]: x are tiles of output rows, w of output columns.
template <class T, bool kAcrossX, bool kAcrossW, int M, int N, int A>
__device__ __forceinline__ void multiply(const i32x4 (&x)[M], const i32x4 (&w)[N], int first, f32x4 (&acc)[A][N]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < M; i++)
#pragma unroll
            for (int j = 0; j < N; j++)
                acc[first + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[j]), __builtin_bit_cast(bf16x8, x[i]),
                                                                            acc[first + i][j], 0, 0, 0);
    } else {
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int i = 0; i < M; i++)
#pragma unroll
                for (int j = 0; j < N; j++)
                    acc[first + i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(element<T, kAcrossW>(w, j, k), element<T, kAcrossX>(x, i, k),
                                                                             acc[first + i][j], 0, 0, 0);
    }
}

// The output row, within a wavefront's rows, of a lane's tile i.
template <class T, bool kAcross, int M>
__device__ __forceinline__ int tile_row(int i) {
    const int i16 = lane_id() & 15;
    return kQuads<T, kAcross, M> ? 64 * (i / 4) + 4 * i16 + i % 4 : 16 * i + i16;
}

// f(column, four values): a lane's outputs of tile row i, four consecutive columns at a time.
template <class T, bool kAcross, int N, class F>
__device__ __forceinline__ void tile_columns(const f32x4 (&acc)[N], const F &f) {
    const int g = lane_id() >> 4;
    if constexpr (kQuads<T, kAcross, N>) {
#pragma unroll
        for (int t = 0; t < N / 4; t++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float v[4] = {acc[4 * t][e], acc[4 * t + 1][e], acc[4 * t + 2][e], acc[4 * t + 3][e]};
                f(64 * t + 16 * g + 4 * e, v);
            }
    } else {
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float v[4] = {acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
            f(16 * j + 4 * g, v);
        }
    }
}

// This wavefront's loads, and its reads of LDS, are done; then the others'.  As
// __syncthreads, but with nothing moved across.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0070);         // vmcnt(0), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// Tiles of output rows that are read together.
template <int M>
constexpr int kGroup = M < 4 ? M : 4;

// The steps of a tile, in two buffers.  fetch_x(step, buffer) and then fetch_w(step, buffer)
// bring a step's sides, store(buffer) puts them where they went through registers, read_x(buffer, h,
// first, x) and read_w(buffer, h, w) take the tiles of 64 bytes h, used(x, first) is shown every
// x once.  Buffers are filled a step ahead; what is multiplied next is read while the tiles
// before it are multiplied, over a step's end too.  Loads are taken no faster than the
// memory's pipe has room, and a wavefront does nothing else until they are: so a step's two sides
// are asked for apart (kApart), with products between, unless both need a look at LDS before that.
//
// Bound by the matrix units at the clocks that the card's power leaves them: 16384 x 4096 x 4096 in
// bfloat16, one type, 414 us, its rows' gradient 416 and its weights' 555, where the library's products take
// 350, 396 and 450.  When it was built, at lower clocks, forward took 493; without its loads 350 to 365, without its
// reads of LDS 420 to 440.  Three and four buffers of half a step each, wavefronts that take turns at multiplying and
// loading, and 4 wavefronts of 128 x 128 outputs measured the same or up to a fifth more.
template <class T, bool kAcrossX, bool kAcrossW, bool kApart, int SB, int M, int N, class Buffer, class FetchX, class FetchW, class Store, class ReadX,
          class ReadW, class Used>
__device__ __forceinline__ void multiply_steps(int steps, const Buffer &buffer, f32x4 (&acc)[M][N], const FetchX &fetch_x,
                                               const FetchW &fetch_w, const Store &store, const ReadX &read_x, const ReadW &read_w,
                                               const Used &used) {
    constexpr int K = kGroup<M>, kGroups = M / K, kParts = SB / 64, kUnits = kParts * kGroups;
    static_assert(kUnits % 2 == 0, "x's two sets of registers take turns over the steps too");
    i32x4 x[2][K], w[2][N];
    fetch_x(0, buffer(0));
    fetch_w(0, buffer(0));
    store(buffer(0));
    meet();
    if (steps > 1) {
        fetch_x(1, buffer(1));
        fetch_w(1, buffer(1));
    }
    read_x(buffer(0), 0, 0, x[0]);
    read_w(buffer(0), 0, w[0]);
    for (int first = 0; first < steps; first += 2) {
        unrolled<2>([&](auto I) {
            constexpr int turn = decltype(I)::value;
            const int step = first + turn;
            if (step >= steps) return;
            unrolled<kUnits>([&](auto U) {
                constexpr int u = decltype(U)::value, next = u + 1, h = u / kGroups;
                if constexpr (next < kUnits) {
                    read_x(buffer(turn), next / kGroups, next % kGroups * K, x[next & 1]);
                    if constexpr (next % kGroups == 0) read_w(buffer(turn), next / kGroups, w[next / kGroups]);
                    // the other side of what the last step began to bring
                    if constexpr (u == 0 && kApart)
                        if (step > 0 && step + 1 < steps) fetch_w(step + 1, buffer(1 - turn));
                } else {
                    if (step + 1 < steps) store(buffer(1 - turn));
                    meet();
                    if (step + 2 < steps) {
                        fetch_x(step + 2, buffer(turn));
                        if constexpr (!kApart) fetch_w(step + 2, buffer(turn));
                    }
                    if (step + 1 < steps) {
                        read_x(buffer(1 - turn), 0, 0, x[0]);
                        read_w(buffer(1 - turn), 0, w[0]);
                    }
                }
                used(x[u & 1], u % kGroups * K);
                multiply<T, kAcrossX, kAcrossW>(x[u & 1], w[h], u % kGroups * K, acc);
            });
        });
    }
}

}  // namespace tgl
