// tgl_typed.hip -- products of rows with their type's weights, and their
// gradients:
//   y[i] = W x[i] + b;  dx[i] = W^T dy[i];  dW = sum dy[i] x[i]^T;  db = sum dy[i]
// over the rows i of a type, whose places are known on the device only: the grid has
// room for as many tiles as there can be, and each finds its type and rows.
#include "tgl_typed.hpp"

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
    float *parts;               // [stretches][out][in] sums of types cut into several, then [stretches][out]
    float *parts_b;
    int64_t dys, xs;
    int32_t out, in;
    int32_t rows;               // of a stretch
    int32_t tiles_in, tiles;    // tiles of dW
    int32_t stretches;          // there is room for
};

constexpr int kTile = 64;
constexpr int kBytes = 128;     // of a tile's row in LDS

__device__ __forceinline__ int swizzle(int r) { return (r >> 1) & 7; }

template <class T>
__device__ __forceinline__ void put_piece(int8_t *tile, int r, int p, const i32x4 &v) {
    *reinterpret_cast<i32x4 *>(tile + r * kBytes + ((p ^ swizzle(r)) * 16)) = v;
}

template <class T>
__device__ __forceinline__ i32x4 get_piece(const int8_t *tile, int r, int p) {
    return *reinterpret_cast<const i32x4 *>(tile + r * kBytes + ((p ^ swizzle(r)) * 16));
}

// kPiece elements that lie across kPiece rows of a tile, at element e of each.
template <class T>
__device__ __forceinline__ void put_across(int8_t *tile, int r, int e, const i32x4 &v) {
    const Run<T, kPiece<T>> x = __builtin_bit_cast(Run<T, kPiece<T>>, v);
#pragma unroll
    for (int i = 0; i < kPiece<T>; i++) {
        const int p = e / kPiece<T>, in = e % kPiece<T>;
        *reinterpret_cast<T *>(tile + (r + i) * kBytes + ((p ^ swizzle(r + i)) * 16) + in * sizeof(T)) = x.t[i];
    }
}

// 64 x 64 outputs of 4 wavefronts, 32 x 32 each; `b` are a tile's output columns.
template <class T>
__device__ __forceinline__ void multiply_tile(const int8_t *a, const int8_t *b, int wm, int wn, f32x4 (&acc)[2][2]) {
    const int i16 = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        i32x4 x[2], w[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            x[i] = get_piece<T>(a, wm * 32 + i * 16 + i16, 4 * h + g);
            w[i] = get_piece<T>(b, wn * 32 + i * 16 + i16, 4 * h + g);
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < 2; j++) acc[i][j] = multiply_pieces<T>(w[j], x[i], acc[i][j]);
    }
}

template <class T, bool kAcross>
__global__ __launch_bounds__(kBlock) void rows_kernel(const RowsArgs a) {
    __shared__ __attribute__((aligned(16))) int8_t at[kTile * kBytes];
    __shared__ __attribute__((aligned(16))) int8_t bt[kTile * kBytes];
    constexpr int kStep = kBytes / sizeof(T), E = kPiece<T>;
    const uint32_t tm = blockIdx.x / a.tiles_n;
    const int n0 = (blockIdx.x % a.tiles_n) * kTile;
    Stretch s;
    if (!find_stretch<true>(a.g, tm, kTile, 0, s)) return;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int i16 = lane & 15, g = lane >> 4, wm = wave >> 1, wn = wave & 1;
    f32x4 acc[2][2] = {};
    if (s.type < a.g.num_types) {
        const T *w = static_cast<const T *>(a.w) + s.type * a.wt;
        const int r0 = threadIdx.x / 8, p = threadIdx.x % 8;        // rows r0 and r0 + 32
        const T *row[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int64_t at = row_at(a.g, s.begin + r0 + 32 * i, s.end);
            row[i] = at < 0 ? nullptr : static_cast<const T *>(a.x) + at * a.xs;
        }
        for (int k0 = 0; k0 < a.k; k0 += kStep) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2; i++) put_piece<T>(at, r0 + 32 * i, p, load_piece(row[i], k0 + p * E, a.k));
            if constexpr (!kAcross) {
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int c = n0 + r0 + 32 * i;
                    put_piece<T>(bt, r0 + 32 * i, p, load_piece(c < a.n ? w + c * a.ws : nullptr, k0 + p * E, a.k));
                }
            } else {
                for (int t = threadIdx.x; t < kStep * (kTile / E); t += kBlock) {
                    const int k = t / (kTile / E), c = t % (kTile / E) * E;
                    put_across<T>(bt, c, k, load_piece(k0 + k < a.k ? w + (k0 + k) * a.ws : nullptr, n0 + c, a.n));
                }
            }
            __syncthreads();
            multiply_tile<T>(at, bt, wm, wn, acc);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int64_t row = row_at(a.g, s.begin + wm * 32 + i * 16 + i16, s.end);
        if (row < 0) continue;
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const int c = n0 + wn * 32 + j * 16 + 4 * g;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                v[e] = acc[i][j][e];
                if (a.bias && s.type < a.g.num_types && c + e < a.n) v[e] += a.bias[static_cast<int64_t>(s.type) * a.n + c + e];
            }
            if (c < a.n) store_columns<T, 4>(static_cast<T *>(a.y) + row * a.ys, c, a.n, v);
        }
    }
}

template <class T>
__global__ __launch_bounds__(kBlock) void sums_kernel(const SumsArgs a) {
    __shared__ __attribute__((aligned(16))) int8_t at[kTile * kBytes];
    __shared__ __attribute__((aligned(16))) int8_t bt[kTile * kBytes];
    constexpr int kStep = kBytes / sizeof(T), E = kPiece<T>;
    const uint32_t stretch = blockIdx.x / a.tiles;
    const int tile = blockIdx.x % a.tiles;
    const int o0 = tile / a.tiles_in * kTile, c0 = tile % a.tiles_in * kTile;
    Stretch s;
    if (!find_stretch<false>(a.g, stretch, a.rows, 1, s)) return;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int i16 = lane & 15, g = lane >> 4, wm = wave >> 1, wn = wave & 1;
    f32x4 acc[2][2] = {};
    float sum = 0.0f;
    for (int64_t p0 = s.begin; p0 < s.end; p0 += kStep) {
        __syncthreads();
        for (int t = threadIdx.x; t < kStep * (kTile / E); t += kBlock) {
            const int k = t / (kTile / E), c = t % (kTile / E) * E;
            const int64_t row = row_at(a.g, p0 + k, s.end);
            put_across<T>(at, c, k, load_piece(row < 0 ? nullptr : static_cast<const T *>(a.dy) + row * a.dys, o0 + c, a.out));
            put_across<T>(bt, c, k, load_piece(row < 0 ? nullptr : static_cast<const T *>(a.x) + row * a.xs, c0 + c, a.in));
        }
        __syncthreads();
        multiply_tile<T>(at, bt, wm, wn, acc);
        if (a.db && c0 == 0 && threadIdx.x < kTile)
            for (int p = 0; p < 8; p++) {
                const Run<T, E> v = __builtin_bit_cast(Run<T, E>, get_piece<T>(at, threadIdx.x, p));
                for (int i = 0; i < E; i++) sum += as_float(v.t[i]);
            }
    }
    const int64_t outs = static_cast<int64_t>(a.out) * a.in;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int o = o0 + wm * 32 + i * 16 + i16;
        if (o >= a.out) continue;
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const int c = c0 + wn * 32 + j * 16 + 4 * g;
            const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (c >= a.in) continue;
            if (s.count == 1) store_columns<T, 4>(static_cast<T *>(a.dw) + s.type * outs + static_cast<int64_t>(o) * a.in, c, a.in, v);
            else store_columns<float, 4>(a.parts + stretch * outs + static_cast<int64_t>(o) * a.in, c, a.in, v);
        }
    }
    if (a.db && c0 == 0 && threadIdx.x < kTile && o0 + static_cast<int>(threadIdx.x) < a.out) {
        const int o = o0 + threadIdx.x;
        if (s.count == 1) a.db[static_cast<int64_t>(s.type) * a.out + o] = sum;
        else a.parts_b[static_cast<int64_t>(stretch) * a.out + o] = sum;
    }
}

// The stretches of a type together, one after another.
template <class T>
__global__ __launch_bounds__(kBlock) void sums_join_kernel(const SumsArgs a, int32_t blocks) {
    const int type = blockIdx.x / blocks;
    // the type's first stretch and their number
    int64_t first = 0;
    int32_t count = 0;
    for (int t = 0; t <= type; t++) {
        int64_t begin = t == 0 ? 0 : a.g.offsets[t], end = a.g.offsets[t + 1];
        begin = begin < 0 ? 0 : begin > a.g.n ? a.g.n : begin;
        end = end > a.g.n ? a.g.n : end < begin ? begin : end;
        first += count;
        count = static_cast<int32_t>((end - begin + a.rows - 1) / a.rows);
        if (count < 1) count = 1;
    }
    if (count == 1 || first + count > a.stretches) return;      // offsets that decrease: nothing to read
    const int64_t outs = static_cast<int64_t>(a.out) * a.in;
    for (int64_t i = static_cast<int64_t>(blockIdx.x % blocks) * kBlock + threadIdx.x; i < outs + (a.db ? a.out : 0);
         i += static_cast<int64_t>(blocks) * kBlock) {
        const float *p = i < outs ? a.parts + first * outs + i : a.parts_b + first * a.out + (i - outs);
        float sum = 0.0f;
        for (int32_t c = 0; c < count; c++) sum += p[c * (i < outs ? outs : a.out)];
        if (i < outs) static_cast<T *>(a.dw)[type * outs + i] = from_float<T>(sum);
        else a.db[static_cast<int64_t>(type) * a.out + (i - outs)] = sum;
    }
}

// Rows of a stretch: as many stretches as give the card two workgroups a unit.
int32_t stretch_rows(int64_t n, int32_t out, int32_t in) {
    const int64_t tiles = static_cast<int64_t>((out + kTile - 1) / kTile) * ((in + kTile - 1) / kTile);
    const int64_t most = (512 + tiles - 1) / tiles;
    int64_t rows = (n + most - 1) / most;
    if (rows < 256) rows = 256;
    return static_cast<int32_t>(rows < (1 << 30) ? (rows + 63) / 64 * 64 : 1 << 30);
}

size_t carve(SumsArgs &a, void *base) {
    Carver c(base);
    const size_t stretches = static_cast<size_t>(a.g.n / a.rows + a.g.num_types);
    if (a.g.n <= a.rows) return 0;              // no type is cut
    a.parts = c.take<float>(stretches * a.out * a.in);
    a.parts_b = c.take<float>(stretches * a.out);
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

template <bool kAcross>
tgl_status launch_rows(const tgl_row_groups *groups, const void *x, int64_t x_stride, const tgl_typed_weights *w,
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
    RowsArgs a{groups_of(groups), x, w->ptr, bias, y, x_stride, w->row_stride, w->type_stride, y_stride, k, n, 0};
    a.tiles_n = (n + kTile - 1) / kTile;
    const int64_t tiles = (groups->n / kTile + groups->num_types + 1) * a.tiles_n;
    if (tiles >= (int64_t(1) << 24)) return TGL_EINVAL;
    if (dtype == TGL_OUT_F32) rows_kernel<float, kAcross><<<static_cast<unsigned>(tiles), kBlock, 0, st>>>(a);
    else rows_kernel<bf16_t, kAcross><<<static_cast<unsigned>(tiles), kBlock, 0, st>>>(a);
    return launch_status();
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_linear_typed(const tgl_row_groups *groups, const void *x, int64_t x_stride,
                            const tgl_typed_weights *w, const float *bias, void *y, int64_t y_stride,
                            int32_t dtype, void *stream) {
    return launch_rows<false>(groups, x, x_stride, w, bias, y, y_stride, dtype, stream);
}

tgl_status tgl_linear_typed_grad_x(const tgl_row_groups *groups, const void *dy, int64_t dy_stride,
                                   const tgl_typed_weights *w, void *dx, int64_t dx_stride, int32_t dtype,
                                   void *stream) {
    return launch_rows<true>(groups, dy, dy_stride, w, nullptr, dx, dx_stride, dtype, stream);
}

size_t tgl_linear_typed_grad_w_workspace(const tgl_row_groups *groups, int32_t out, int32_t in, int32_t dtype) {
    if (!groups || groups->n < 0 || groups->num_types < 1 || !valid_dims(out, in) || !is_elem_type(dtype)) return 0;
    SumsArgs a{};
    a.g = groups_of(groups);
    a.out = out;
    a.in = in;
    a.rows = stretch_rows(a.g.n, out, in);
    return carve(a, nullptr);
}

tgl_status tgl_linear_typed_grad_w(const tgl_row_groups *groups, const void *dy, int64_t dy_stride, const void *x,
                                   int64_t x_stride, int32_t out, int32_t in, void *dw, float *db, int32_t dtype,
                                   void *workspace, size_t workspace_bytes, void *stream) {
    if (!valid_groups(groups) || !valid_dims(out, in) || !is_elem_type(dtype)) return TGL_EINVAL;
    const size_t e = elem_size(dtype);
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dw, e) || !aligned(db, 4) || !dw) return TGL_EINVAL;
    if (groups->n > 0 && (!dy || !x)) return TGL_EINVAL;
    SumsArgs a{groups_of(groups), dy, x, dw, db, nullptr, nullptr, dy_stride, x_stride, out, in, 0, 0, 0, 0};
    a.rows = stretch_rows(a.g.n, out, in);
    const size_t need = carve(a, nullptr);
    if (need) {
        if (!workspace || workspace_bytes < need) return TGL_ENOSPACE;
        if (!aligned(workspace, 256)) return TGL_EINVAL;
        carve(a, workspace);
    }
    a.tiles_in = (in + kTile - 1) / kTile;
    a.tiles = (out + kTile - 1) / kTile * a.tiles_in;
    a.stretches = static_cast<int32_t>(a.g.n / a.rows + a.g.num_types);
    const int64_t grid = static_cast<int64_t>(a.stretches) * a.tiles;
    if (grid >= (int64_t(1) << 24)) return TGL_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (dtype == TGL_OUT_F32) sums_kernel<float><<<static_cast<unsigned>(grid), kBlock, 0, st>>>(a);
    else sums_kernel<bf16_t><<<static_cast<unsigned>(grid), kBlock, 0, st>>>(a);
    if (!need || launch_status() != TGL_OK) return launch_status();
    const int32_t blocks = 64;
    const unsigned join = static_cast<unsigned>(a.g.num_types) * blocks;
    if (dtype == TGL_OUT_F32) sums_join_kernel<float><<<join, kBlock, 0, st>>>(a, blocks);
    else sums_join_kernel<bf16_t><<<join, kBlock, 0, st>>>(a, blocks);
    return launch_status();
}

}  // extern "C"
