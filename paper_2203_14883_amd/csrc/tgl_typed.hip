// tgl_typed.hip -- products of rows with their type's weights, and their
// gradients:
//   y[i] = W x[i] + b;  dx[i] = W^T dy[i];  dW = sum dy[i] x[i]^T;  db = sum dy[i]
// over the rows i of a type, whose places are known on the device only: the grid has
// room for as many tiles as there can be, and each finds its type and rows.
#include <type_traits>

#include "tgl_typed_tile.hpp"

namespace tgl {
namespace {

struct RowsArgs {               // y and dx
    Groups g;
    const void *x;
    const void *w;
    const float *bias;
    void *y;
    int64_t xs, ws, wt, ys;     // row strides of x, w, y; type stride of w
    int32_t k, n;               // the sum's axis; columns of y
    int32_t tiles_n;
};

struct SumsArgs {               // dW and db
    Groups g;
    const void *dy;
    const void *x;
    void *dw;
    float *db;
    float *parts;               // [room][out][in] sums of the stretches of types that are cut into several
    double *parts_b;            // [room][out]
    int64_t dys, xs;
    int32_t out, in;
    int32_t rows;               // of a stretch
    int32_t tile;
    int32_t tiles_in, tiles;    // tiles of dW
    uint32_t stretches;         // at most
    uint32_t room;              // of those of types that are cut, at most
};

// Tile `id` of rows x cols, in bands of `band` rows walked column by column, so
// that tiles of neighbouring numbers share what they read.
__device__ __forceinline__ void banded(uint32_t id, uint32_t rows, uint32_t cols, uint32_t band, uint32_t &r, uint32_t &c) {
    const uint32_t b = id / (band * cols), in = id - b * band * cols;
    const uint32_t left = rows - b * band, height = left < band ? left : band;
    c = in / height;
    r = b * band + (in - c * height);
}

// A workgroup's number among `work` pieces of work: the 8 dies take workgroups in
// turn, and each gets a contiguous stretch.  False if there is none for it; `at`, the
// workgroup's number within its die, then is the number among those that come after.
__device__ __forceinline__ bool die_major(uint32_t work, uint32_t &at, uint32_t &id) {
    const uint32_t per = (work + 7) / 8;
    id = (blockIdx.x & 7) * per + at;
    at = at < per ? ~0u : at - per;
    return at == ~0u && id < work;
}

// Zeros for a tile of the rows of no type.
template <class T, int BM, int BN>
__device__ __forceinline__ void clear_tile(const RowsArgs &a, int64_t begin, int n0) {
    constexpr float kNone[4] = {};
    const int cols = a.n - n0 < BN ? a.n - n0 : BN;
    for (int i = threadIdx.x; i < BM * (BN / 4); i += blockDim.x) {
        const int64_t row = row_at(a.g, begin + i / (BN / 4), a.g.n);
        const int c = i % (BN / 4) * 4;
        if (row >= 0 && c < cols) store_columns<T, 4>(static_cast<T *>(a.y) + row * a.ys, n0 + c, a.n, kNone);
    }
}

// ROWS rows of one type, BM of them at most, times BN columns; a wavefront has 64 columns.
template <class T, bool kAcross, int ROWS, int BM, int BN, int NW, int SB, bool kDirect>
__device__ __forceinline__ void rows_tile(const RowsArgs &a, const Stretch &s, int n0, int8_t (&steps_of)[2][(BM + BN) * SB]) {
    constexpr int kWaveN = BN / 64, MT = ROWS / (NW / kWaveN) / 16, NT = 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / kWaveN, wn = wave % kWaveN;
    f32x4 acc[MT][NT] = {};
    using X = Along<T, ROWS, NW, SB, kDirect>;
    using W = std::conditional_t<kAcross, Across<T, BN, NW, SB, kDirect>, Along<T, BN, NW, SB, kDirect>>;
    {
        X x;
        W w;
        x.length = a.k;
        int32_t row[X::kFetch];
        rows_at(a.g, s.end, [&](int f) { return s.begin + X::edge(wave, f); }, row);
#pragma unroll
        for (int f = 0; f < X::kFetch; f++) x.set(wave, f, static_cast<const T *>(a.x) + (row[f] < 0 ? 0 : row[f]) * a.xs);
        const T *weights = static_cast<const T *>(a.w) + s.type * a.wt;
        if constexpr (kAcross) {
            w.set(wave, weights, a.ws, a.k, n0, a.n);
        } else {
            w.length = a.k;
#pragma unroll
            for (int f = 0; f < W::kFetch; f++) {
                const int c = n0 + W::edge(wave, f);
                w.set(wave, f, weights + (c < a.n ? c : a.n - 1) * a.ws);
            }
        }
        multiply_steps<T, false, kAcross, true, SB>(
            (a.k + kStep<T, SB> - 1) / kStep<T, SB>, [&](int i) { return steps_of[i]; }, acc,
            [&](int step, int8_t *buf) { x.fetch(wave, step, buf); },
            [&](int step, int8_t *buf) { w.fetch(wave, step, buf + BM * SB); },
            [&](int8_t *buf) {
                x.store(wave, buf);
                w.store(wave, buf + BM * SB);
            },
            [&](const int8_t *buf, int h, int first, auto &v) { X::read(buf, 0, (wm * MT + first) * 16, h, v); },
            [&](const int8_t *buf, int h, i32x4(&v)[NT]) { W::read(buf, BM * SB, wn * 64, h, v); }, [](const auto &, int) {});
    }
    const float *bias = a.bias ? a.bias + static_cast<int64_t>(s.type) * a.n : nullptr;
    int32_t row[MT];
    rows_at(a.g, s.end, [&](int i) { return s.begin + wm * MT * 16 + tile_row<T, false, MT>(i); }, row);
#pragma unroll
    for (int i = 0; i < MT; i++) {
        if (row[i] < 0) continue;
        T *y = static_cast<T *>(a.y) + row[i] * a.ys;
        tile_columns<T, kAcross>(acc[i], [&](int c, const float(&v)[4]) {
            const int col = n0 + wn * 64 + c;
            if (col >= a.n) return;
            float out[4] = {v[0], v[1], v[2], v[3]};
            if (bias) {
                float b[4];
                load_columns<float, 4>(bias, col, a.n, b);
#pragma unroll
                for (int e = 0; e < 4; e++) out[e] += b[e];
            }
            store_columns<T, 4>(y, col, a.n, out);
        });
    }
}

template <class T, bool kAcross, int BM, int BN, int NW, int SB, bool kDirect>
__global__ __launch_bounds__(NW * kWave, 2) void rows_kernel(const RowsArgs a) {
    __shared__ __attribute__((aligned(1024))) int8_t steps_of[2][(BM + BN) * SB];
    uint32_t at = blockIdx.x >> 3, id, tm, tn;
    Stretches cut(a.g, BM, 0, 0);
    const uint32_t tiles_m = cut.all();
    if (!die_major(tiles_m * a.tiles_n, at, id)) {
        // rows of no type, which every die has its part of
        const int64_t begin = typed_rows(a.g);
        const uint32_t clear = static_cast<uint32_t>((a.g.n - begin + BM - 1) / BM) * a.tiles_n;
        if (at != ~0u && die_major(clear, at, id))
            clear_tile<T, BM, BN>(a, begin + static_cast<int64_t>(id / a.tiles_n) * BM, id % a.tiles_n * BN);
        return;
    }
    banded(id, tiles_m, a.tiles_n, 8, tm, tn);
    Stretch s;
    if (!cut.find(tm, s)) return;
    // a type's last rows fill half a tile as often as not: half the products then (16,384 rows of 8 types, 4096
    // x 4096 in bfloat16: 68 tiles of rows where 64 would do, 646 us without)
    if constexpr (BM == 256) {
        if (s.end - s.begin <= BM / 2) {
            rows_tile<T, kAcross, BM / 2, BM, BN, NW, SB, kDirect>(a, s, tn * BN, steps_of);
            return;
        }
    }
    rows_tile<T, kAcross, BM, BM, BN, NW, SB, kDirect>(a, s, tn * BN, steps_of);
}

// Few rows: a workgroup per 16 rows of a type and 16 columns, operands straight
// from memory (kAcross: the weights element by element, 16 columns of a row of memory at a
// time).  Its wavefronts take pieces of the sum's axis in turn and add up through LDS, in
// their order.  Bound by latency where the weights are small (a row of 768 -> 2304 bfloat16 4.0 us, in
// tiles of 64 7.9) and by their bytes where they are not.
template <class T, bool kAcross, int NW>
__global__ __launch_bounds__(NW * kWave) void rows_few_kernel(const RowsArgs a) {
    __shared__ f32x4 sums[NW][kWave];
    constexpr int kAhead = 4;                   // pieces of a lane on their way
    Stretches cut(a.g, 16, 0, 0);
    const uint32_t tiles_m = cut.all(), tm = blockIdx.x / a.tiles_n;
    const int n0 = static_cast<int>(blockIdx.x - tm * a.tiles_n) * 16;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (tm >= tiles_m) {
        const int64_t begin = typed_rows(a.g) + static_cast<int64_t>(tm - tiles_m) * 16;
        if (begin < a.g.n) clear_tile<T, 16, 16>(a, begin, n0);
        return;
    }
    Stretch s;
    if (!cut.find(tm, s)) return;
    int32_t row[1];
    rows_at(a.g, s.end, [&](int) { return s.begin + (lane & 15); }, row);
    const T *x = static_cast<const T *>(a.x) + (row[0] < 0 ? 0 : row[0]) * a.xs;
    const int c = n0 + (lane & 15);
    const T *w = static_cast<const T *>(a.w) + s.type * a.wt + (c < a.n ? c : a.n - 1) * (kAcross ? 1 : a.ws);
    constexpr int E = kPiece<T>, kLength = 4 * E;               // of the sum's axis that a wavefront takes at a time
    using word_t = i32x4 __attribute__((aligned(alignof(T))));
    f32x4 acc[1][1] = {};
    auto weights = [&](int k, bool whole) {
        if constexpr (kAcross) {
            Run<T, E> v = {};
#pragma unroll
            for (int i = 0; i < E; i++)
                if (whole || k + i < a.k) v.t[i] = w[(k + i) * a.ws];
            return __builtin_bit_cast(i32x4, v);
        } else {
            return whole ? static_cast<i32x4>(*reinterpret_cast<const word_t *>(w + k)) : load_piece(w, k, a.k);
        }
    };
    const int own = (lane >> 4) * E;
    int k = wave * kLength;
    for (; k + (kAhead - 1) * NW * kLength + kLength <= a.k; k += kAhead * NW * kLength) {
        i32x4 xv[kAhead][1], wv[kAhead][1];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            wv[u][0] = weights(k + own + u * NW * kLength, true);
            xv[u][0] = *reinterpret_cast<const word_t *>(x + k + own + u * NW * kLength);
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++) multiply<T, false, false>(xv[u], wv[u], 0, acc);
    }
    for (; k < a.k; k += NW * kLength) {
        const i32x4 xv[1] = {load_piece(x, k + own, a.k)}, wv[1] = {weights(k + own, false)};
        multiply<T, false, false>(xv, wv, 0, acc);
    }
    sums[wave][lane] = acc[0][0];
    __syncthreads();
    if (wave != 0 || row[0] < 0) return;
    f32x4 sum = sums[0][lane];
#pragma unroll
    for (int i = 1; i < NW; i++) sum += sums[i][lane];
    const int col = n0 + 4 * (lane >> 4);
    if (col >= a.n) return;
    float out[4] = {sum[0], sum[1], sum[2], sum[3]};
    if (a.bias) {
        float b[4];
        load_columns<float, 4>(a.bias + static_cast<int64_t>(s.type) * a.n, col, a.n, b);
#pragma unroll
        for (int e = 0; e < 4; e++) out[e] += b[e];
    }
    store_columns<T, 4>(static_cast<T *>(a.y) + row[0] * a.ys, col, a.n, out);
}

// BM rows times BN columns of dW, over a stretch of a type's rows.
template <class T, int BM, int BN, int NW, int SB, bool kDirect>
__global__ __launch_bounds__(NW * kWave, 2) void sums_kernel(const SumsArgs a) {
    constexpr int kWaveN = BN / 64, MT = BM / (NW / kWaveN) / 16, NT = 4;
    __shared__ __attribute__((aligned(1024))) int8_t steps_of[2][(BM + BN) * SB];
    // A stretch's tiles, which read the same rows, go to one die.  Many stretches, whose lengths differ, go to the
    // dies in turn; few are cut into tiles for all dies.
    uint32_t at = blockIdx.x >> 3, stretch, tile, to, ti;
    Stretches cut(a.g, a.rows, 1, kStep<T, SB>);
    if (a.stretches >= 64) {
        stretch = at / a.tiles * 8 + (blockIdx.x & 7);
        tile = at % a.tiles;
        if (stretch >= a.stretches) return;
        if (a.g.num_types <= kWave) cut.take(0);
    } else {
        const uint32_t stretches = cut.all();
        uint32_t id;
        if (!die_major((stretches < a.stretches ? stretches : a.stretches) * a.tiles, at, id)) return;
        stretch = id / a.tiles;
        tile = id - stretch * a.tiles;
    }
    banded(tile, a.tiles / a.tiles_in, a.tiles_in, 4, to, ti);
    const int o0 = to * BM, c0 = ti * BN;
    Stretch s;
    if (!cut.find(stretch, s) || (s.count > 1 && s.part >= a.room)) return;     // (offsets that decrease)
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / kWaveN, wn = wave % kWaveN;
    f32x4 acc[MT][NT] = {};
    constexpr int kSums = (MT + kWaveN - 1) / kWaveN;
    // Of dy, tiles wn, wn + kWaveN, ... of the wavefront's rows: 4 or 8 places at a time in 32 bits, beyond that in 64.  In 32
    // alone a lane's sum over 16,384 places of one number is off by 1.5e-4 of it; the time is the same.
    double sum[kSums] = {};
    const bool want_sum = a.db && ti == 0;
    using D = Gathered<T, BM, NW, SB, kDirect>;
    using X = Gathered<T, BN, NW, SB, kDirect>;
    if (s.end > s.begin) {
        D d;
        X x;
        d.set(static_cast<const T *>(a.dy), a.dys, o0, a.out);
        x.set(static_cast<const T *>(a.x), a.xs, c0, a.in);
        Places<kStep<T, SB> / NW> places(a.g, s.begin, s.end, wave * (kStep<T, SB> / NW));
        multiply_steps<T, true, true, false, SB>(
            static_cast<int>((s.end - s.begin + kStep<T, SB> - 1) / kStep<T, SB>), [&](int i) { return steps_of[i]; }, acc,
            [&](int, int8_t *buf) {
                places.advance(kStep<T, SB>);
                d.fetch(wave, places, buf);
            },
            [&](int, int8_t *buf) {
                x.fetch(wave, places, buf + BM * SB);
                places.load();
            },
            [&](int8_t *buf) {
                d.store(wave, buf);
                x.store(wave, buf + BM * SB);
            },
            [&](const int8_t *buf, int h, int first, auto &v) { D::read(buf, 0, (wm * MT + first) * 16, h, v); },
            [&](const int8_t *buf, int h, i32x4(&v)[NT]) { X::read(buf, BM * SB, wn * 64, h, v); },
            [&](const auto &dv, int first) {
                if (!want_sum) return;
#pragma unroll
                for (int i = 0; i < kGroup<MT>; i++) {
                    if (i % kWaveN != wn) continue;             // first is a multiple of 4, or 0
                    float v = 0.0f;
                    if constexpr (sizeof(T) == 2) {
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            v += __builtin_bit_cast(float, dv[i][e] << 16);
                            v += __builtin_bit_cast(float, dv[i][e] & static_cast<int>(0xffff0000u));
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; e++) v += element<T, true>(dv, i, e);
                    }
                    sum[(first + i) / kWaveN] += v;
                }
            });
    }
    const int64_t outs = static_cast<int64_t>(a.out) * a.in;
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int o = o0 + wm * MT * 16 + tile_row<T, true, MT>(i);
        if (want_sum && i % kWaveN == wn) {
            double v = sum[i / kWaveN];
            v += __shfl_xor(v, 16, kWave);
            v += __shfl_xor(v, 32, kWave);
            if (lane < 16 && o < a.out) {
                if (s.count == 1) a.db[static_cast<int64_t>(s.type) * a.out + o] = static_cast<float>(v);
                else a.parts_b[static_cast<int64_t>(s.part) * a.out + o] = v;
            }
        }
        if (o >= a.out) continue;
        tile_columns<T, true>(acc[i], [&](int c, const float(&v)[4]) {
            const int col = c0 + wn * 64 + c;
            if (col >= a.in) return;
            if (s.count == 1) store_columns<T, 4>(static_cast<T *>(a.dw) + s.type * outs + static_cast<int64_t>(o) * a.in, col, a.in, v);
            else store_columns<float, 4>(a.parts + s.part * outs + static_cast<int64_t>(o) * a.in, col, a.in, v);
        });
    }
}

// The stretches of a type together, one after another, in 64 bits (which costs nothing beside their reading, and a hundred
// of them in 32 lose more than a stretch does): four outputs a thread.
template <class T>
__global__ __launch_bounds__(kBlock) void sums_join_kernel(const SumsArgs a, uint32_t blocks) {
    const int type = blockIdx.x / blocks;
    int64_t first;
    const int32_t count = Stretches(a.g, a.rows, 1, 1).of_type(type, first);
    if (count == 1 || first + count > a.room) return;      // offsets that decrease: nothing to read
    const int64_t outs = static_cast<int64_t>(a.out) * a.in;
    const int64_t own = static_cast<int64_t>(blockIdx.x % blocks) * kBlock + threadIdx.x, step = static_cast<int64_t>(blocks) * kBlock;
    for (int64_t i = own * 4; i < outs; i += step * 4) {
        double sum[4] = {};
        // as many loads on their way as there are registers for
#pragma unroll 8
        for (int32_t c = 0; c < count; c++) {
            float v[4];
            load_columns<float, 4>(a.parts + (first + c) * outs + i, 0, outs - i < 4 ? static_cast<int>(outs - i) : 4, v);
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += v[e];
        }
        const float joined[4] = {static_cast<float>(sum[0]), static_cast<float>(sum[1]), static_cast<float>(sum[2]), static_cast<float>(sum[3])};
        store_columns<T, 4>(static_cast<T *>(a.dw) + type * outs + i, 0, outs - i < 4 ? static_cast<int>(outs - i) : 4, joined);
    }
    if (!a.db) return;
    for (int64_t o = own; o < a.out; o += step) {
        double sum = 0.0;
#pragma unroll 8
        for (int32_t c = 0; c < count; c++) sum += a.parts_b[(first + c) * a.out + o];
        a.db[static_cast<int64_t>(type) * a.out + o] = static_cast<float>(sum);
    }
}

// The tiles of a call's outputs in bfloat16: the largest of which there are still enough.  us
// of tiles of 256 / 128 / 64: 132,000 rows of 768 -> 256 90 / - / 121, 12,000 of 768 -> 1024 33 / 35 / 43, 20,000 of 16 types
// 58 / - / 73, 40,000 of 272 -> 128 - / 14 / 15.
int tile_of(int64_t rows, int64_t cols) {
    auto tiles = [&](int64_t t) { return (rows + t - 1) / t * ((cols + t - 1) / t); };
    return tiles(256) >= 160 ? 256 : tiles(128) >= 256 ? 128 : 64;
}

// dW: its tiles, and the rows of a stretch, of which there are as many as fill the card.
void plan_sums(SumsArgs &a, int32_t dtype) {
    const bool wide = dtype == TGL_OUT_BF16 && a.out >= 192 && a.in >= 192 && a.g.n / a.g.num_types >= 2048;
    a.tile = wide ? 256 : dtype == TGL_OUT_BF16 && a.out > 64 && a.in > 64 && a.g.n / a.g.num_types >= 512 ? 128 : 64;
    a.tiles_in = (a.in + a.tile - 1) / a.tile;
    a.tiles = (a.out + a.tile - 1) / a.tile * a.tiles_in;
    const int64_t target = a.tile == 256 ? 512 : a.tile == 128 ? 1024 : 2560;        // twice what runs at a time
    const int64_t most = (target + a.tiles - 1) / a.tiles;
    int64_t rows = (a.g.n + most - 1) / most;
    if (rows < 256) rows = 256;
    a.rows = static_cast<int32_t>(rows < (1 << 30) ? (rows + 63) / 64 * 64 : 1 << 30);
    a.stretches = static_cast<uint32_t>(a.g.n / a.rows + a.g.num_types);
    a.room = static_cast<uint32_t>(2 * (a.g.n / a.rows));       // a type of more than `rows` has fewer than twice its share
}

size_t carve(SumsArgs &a, void *base) {
    Carver c(base);
    if (a.g.n <= a.rows) return 0;              // no type is cut
    a.parts = c.take<float>(static_cast<size_t>(a.room) * a.out * a.in);
    a.parts_b = c.take<double>(static_cast<size_t>(a.room) * a.out);
    return c.size();
}

bool valid_groups(const tgl_row_groups *g) {
    return g && g->n >= 0 && g->n < (int64_t(1) << 31) && g->num_types >= 1 && g->num_types <= TGL_MAX_TYPES &&
           g->reserved == 0 && g->offsets && aligned(g->offsets, 8) && aligned(g->order, 4);
}

bool valid_dims(int32_t out, int32_t in) {
    return out >= 1 && out <= TGL_MAX_TYPED_DIM && in >= 1 && in <= TGL_MAX_TYPED_DIM;
}

Groups groups_of(const tgl_row_groups *g) { return Groups{g->order, g->offsets, g->n, g->num_types}; }

bool wide_rows(const void *p, int64_t stride, size_t e) { return aligned(p, 16) && stride * static_cast<int64_t>(e) % 16 == 0; }

// Types that can have rows.  Tiles of t rows are n / t and one for each of these and for the rows of no type at most.
int64_t filled_types(const Groups &g) { return g.n < g.num_types ? g.n : g.num_types; }

constexpr int kStepBytes = 128;                         // of the sum's axis
template <int NW>
constexpr int64_t kMostBlocks = ((int64_t(1) << 32) - 1) / (NW * kWave);     // of a launch, whose threads are fewer than 2^32

template <class T, bool kAcross, int B, int NW, bool kDirect>
tgl_status launch_rows(RowsArgs a, hipStream_t st) {
    a.tiles_n = (a.n + B - 1) / B;
    const int64_t work = (a.g.n / B + filled_types(a.g) + 1) * a.tiles_n + 8;        // a die rounds up twice
    if (work + 8 > kMostBlocks<NW>) return TGL_EINVAL;
    rows_kernel<T, kAcross, B, B, NW, kStepBytes, kDirect><<<static_cast<unsigned>((work + 7) / 8 * 8), NW * kWave, 0, st>>>(a);
    return launch_status();
}

// Whether a call is too small for tiles of 64, by its tiles of 16: up to 900 of them (less time at 805 and 896, more at 1024)
// however long the sum's axis; in float32, whose products take long, also where they cover half of what tiles of 64
// would, as those of many types with few rows.  us of tiles of 64 / 16: bfloat16 65 x 768 x 1024 of 4 types 7.7 / 5.4, 1801
// x 272 x 100 of 3 5.1 / 4.4, 200 x 768 x 1024 of 4 7.9 / 8.4, of 64 17 / 22; float32 19.9 / 8.1, 9.4 / 5.7, 20 / 13.8, 70 / 37,
// 1000 x 768 x 768 of 3 23 / 39.  Long axes, of one type: bfloat16 190 x 16,384 x 1024 148 / 87, 190 x 65,536 x 1024 593 / 337, 3500 x
// 16,384 x 64 138 / 115; float32 388 / 170, 2048 / 699, 385 / 226.  Weights across the sum's axis, bfloat16: 64 x 16,384 x 1024
// 162 / 40, 890 x 8192 x 256 81 / 58, but 190 x 768 x 1024 8.5 / 12.3.
bool few_rows(const RowsArgs &a, size_t e) {
    auto tiles = [&](int64_t t) { return (a.g.n / t + filled_types(a.g)) * ((a.n + t - 1) / t); };
    return tiles(16) <= 900 || (e == 4 && tiles(16) <= 8192 && 2 * tiles(16) <= 16 * tiles(64));
}

template <class T, bool kAcross>
tgl_status launch_few(RowsArgs a, hipStream_t st) {
    a.tiles_n = (a.n + 15) / 16;
    const unsigned grid = static_cast<unsigned>((a.g.n / 16 + filled_types(a.g) + 1) * a.tiles_n);
    if (a.k * sizeof(T) <= 512) rows_few_kernel<T, kAcross, 4><<<grid, 4 * kWave, 0, st>>>(a);
    else rows_few_kernel<T, kAcross, 8><<<grid, 8 * kWave, 0, st>>>(a);
    return launch_status();
}

template <class T, bool kAcross>
tgl_status launch_rows(const RowsArgs &a, bool direct, hipStream_t st) {
    if (few_rows(a, sizeof(T))) return launch_few<T, kAcross>(a, st);
    // float32's products take 16 times as long as bfloat16's, so loads are no matter and the smallest tiles waste least:
    // 120,000 rows of 272 -> 128 in tiles of 64 98 us, of 128 112; 40,000 of 272 -> 100 47 and 55
    if constexpr (sizeof(T) == 2) {
        const int tile = tile_of(a.g.n, a.n);
        if (tile == 256 && direct) return launch_rows<T, kAcross, 256, 8, true>(a, st);
        if (tile >= 128) return direct ? launch_rows<T, kAcross, 128, 4, true>(a, st) : launch_rows<T, kAcross, 128, 4, false>(a, st);
    }
    return direct ? launch_rows<T, kAcross, 64, 4, true>(a, st) : launch_rows<T, kAcross, 64, 4, false>(a, st);
}

template <bool kAcross>
tgl_status rows_call(const tgl_row_groups *groups, const void *x, int64_t x_stride, const tgl_typed_weights *w,
                     const float *bias, void *y, int64_t y_stride, int32_t dtype, void *stream) {
    if (!valid_groups(groups) || !w || !valid_dims(w->out, w->in) || !is_elem_type(dtype) || w->row_stride < w->in)
        return TGL_EINVAL;
    const size_t e = elem_size(dtype);
    const int32_t n = kAcross ? w->in : w->out, k = kAcross ? w->out : w->in;
    if (!aligned(x, e) || !aligned(y, e) || !aligned(w->ptr, e) || !aligned(bias, 4)) return TGL_EINVAL;
    if (groups->n > 0 && (!x || !y || !w->ptr || (groups->n > 1 && y_stride < n))) return TGL_EINVAL;
    if (groups->n == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const RowsArgs a{groups_of(groups), x, w->ptr, bias, y, x_stride, w->row_stride, w->type_stride, y_stride, k, n, 0};
    const bool direct = wide_rows(x, x_stride, e) && wide_rows(w->ptr, w->row_stride, e) && w->type_stride * e % 16 == 0 &&
                        k * e % 16 == 0 && (!kAcross || (n * e % 16 == 0 && w->row_stride < (1 << 26)));
    return dtype == TGL_OUT_F32 ? launch_rows<float, kAcross>(a, direct, st) : launch_rows<bf16_t, kAcross>(a, direct, st);
}

template <class T, int B, int NW, bool kDirect>
tgl_status launch_sums(const SumsArgs &a, hipStream_t st) {
    const int64_t work = (static_cast<int64_t>(a.stretches) + 7) / 8 * 8 * a.tiles;
    if (work + 8 > kMostBlocks<NW>) return TGL_EINVAL;
    sums_kernel<T, B, B, NW, kStepBytes, kDirect><<<static_cast<unsigned>(work), NW * kWave, 0, st>>>(a);
    return launch_status();
}

template <class T>
tgl_status launch_sums(const SumsArgs &a, bool direct, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (a.tile == 256) return launch_sums<T, 256, 8, true>(a, st);
        if (a.tile == 128) return direct ? launch_sums<T, 128, 4, true>(a, st) : launch_sums<T, 128, 4, false>(a, st);
    }
    return direct ? launch_sums<T, 64, 4, true>(a, st) : launch_sums<T, 64, 4, false>(a, st);
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_linear_typed(const tgl_row_groups *groups, const void *x, int64_t x_stride,
                            const tgl_typed_weights *w, const float *bias, void *y, int64_t y_stride,
                            int32_t dtype, void *stream) {
    return rows_call<false>(groups, x, x_stride, w, bias, y, y_stride, dtype, stream);
}

tgl_status tgl_linear_typed_grad_x(const tgl_row_groups *groups, const void *dy, int64_t dy_stride,
                                   const tgl_typed_weights *w, void *dx, int64_t dx_stride, int32_t dtype,
                                   void *stream) {
    return rows_call<true>(groups, dy, dy_stride, w, nullptr, dx, dx_stride, dtype, stream);
}

size_t tgl_linear_typed_grad_w_workspace(const tgl_row_groups *groups, int32_t out, int32_t in, int32_t dtype) {
    if (!groups || groups->n < 0 || groups->num_types < 1 || !valid_dims(out, in) || !is_elem_type(dtype)) return 0;
    SumsArgs a{};
    a.g = groups_of(groups);
    a.out = out;
    a.in = in;
    plan_sums(a, dtype);
    return carve(a, nullptr);
}

tgl_status tgl_linear_typed_grad_w(const tgl_row_groups *groups, const void *dy, int64_t dy_stride, const void *x,
                                   int64_t x_stride, int32_t out, int32_t in, void *dw, float *db, int32_t dtype,
                                   void *workspace, size_t workspace_bytes, void *stream) {
    if (!valid_groups(groups) || !valid_dims(out, in) || !is_elem_type(dtype)) return TGL_EINVAL;
    const size_t e = elem_size(dtype);
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dw, e) || !aligned(db, 4) || !dw) return TGL_EINVAL;
    if (groups->n > 0 && (!dy || !x)) return TGL_EINVAL;
    SumsArgs a{};
    a.g = groups_of(groups);
    a.dy = dy;
    a.x = x;
    a.dw = dw;
    a.db = db;
    a.dys = dy_stride;
    a.xs = x_stride;
    a.out = out;
    a.in = in;
    plan_sums(a, dtype);
    const bool direct = wide_rows(dy, dy_stride, e) && wide_rows(x, x_stride, e) && out * e % 16 == 0 && in * e % 16 == 0;
    if (!direct && a.tile == 256) {             // 128 through registers
        a.tile = 128;
        a.tiles_in = (in + 127) / 128;
        a.tiles = (out + 127) / 128 * a.tiles_in;
    }
    const size_t need = carve(a, nullptr);
    if (need) {
        if (!workspace || workspace_bytes < need) return TGL_ENOSPACE;
        if (!aligned(workspace, 256)) return TGL_EINVAL;
        carve(a, workspace);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const tgl_status done = dtype == TGL_OUT_F32 ? launch_sums<float>(a, direct, st) : launch_sums<bf16_t>(a, direct, st);
    if (!need || done != TGL_OK) return done;
    // a workgroup for every 1024 outputs of a type, 4096 in all: most types are not cut
    const int64_t each = (static_cast<int64_t>(out) * in + 1023) / 1024, most = (4096 + a.g.num_types - 1) / a.g.num_types;
    const uint32_t blocks = static_cast<uint32_t>(each < most ? each : most);
    const unsigned join = static_cast<unsigned>(a.g.num_types) * blocks;
    if (dtype == TGL_OUT_F32) sums_join_kernel<float><<<join, kBlock, 0, st>>>(a, blocks);
    else sums_join_kernel<bf16_t><<<join, kBlock, 0, st>>>(a, blocks);
    return launch_status();
}

}  // extern "C"
