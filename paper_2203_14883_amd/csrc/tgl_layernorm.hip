// tgl_layernorm.hip -- residual addition and layer norm of rows, and their
// gradients.
//
//   h = x + r;  m = mean(h);  s = 1 / sqrt(mean((h - m)^2) + eps);  y = (h - m) s w + b
//   xh = (h - m) s;  g = dy w;  dx = (g - mean(g) - xh mean(g xh)) s + dh
//   dw = sum dy xh;  db = sum dy
//
// A row is read once and stays in the registers of L lanes, so the mean of the
// squared distances is taken from the distances themselves.  Sums, and
// distances before they are scaled, are of 64 bits: squares of finite float32
// numbers leave that type's range, and a mean that is large beside the
// distances would lose their bits in 32.  The card does 64-bit sums and
// products at the rate of float32's, and memory bounds these kernels.
#include "tgl_int8.hpp"

namespace tgl {
namespace {

constexpr int kRun = 8;             // elements of a lane's access

struct NormArgs {
    const void *x;
    const void *r;
    const float *w;
    const float *b;
    void *y;
    void *sum;
    double *stats;
    int64_t xs, rs, ys, ss;
    int64_t n;
    int32_t dim;
    float eps;
};

struct GradArgs {
    const void *dy;
    const void *h;
    const void *dh;
    const double *stats;
    const float *w;
    void *dx;
    double *parts;          // [workgroups][2][dim]: each one's sums of dy xh and of dy
    int64_t dys, hs, dhs, dxs;
    int64_t n;
    int32_t dim;
};

// Sum over the L lanes of a row, in all of them.  `lds` has one number per wavefront of
// the workgroup and is free again after the next barrier.
template <int L, int N>
__device__ __forceinline__ void row_sum(double (&v)[N], double (*lds)[N]) {
#pragma unroll
    for (int d = (L < kWave ? L : kWave) / 2; d >= 1; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], d, kWave);
    if constexpr (L > kWave) {
        constexpr int kWaves = L / kWave;
        const int wave = threadIdx.x / kWave, first = wave / kWaves * kWaves;
        if (lane_id() == 0)
            for (int i = 0; i < N; i++) lds[wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; i++) {
            v[i] = 0.0;
#pragma unroll
            for (int k = 0; k < kWaves; k++) v[i] += lds[first + k][i];
        }
    }
}

// A lane's columns of the weights (or what stands for none).
template <int L, int H>
__device__ __forceinline__ void load_weights(const float *w, int i, int runs, int dim, float without, float (&v)[H][kRun]) {
#pragma unroll
    for (int h = 0; h < H; h++) {
#pragma unroll
        for (int k = 0; k < kRun; k++) v[h][k] = without;
        if (w && i + h * L < runs) load_columns<float, kRun>(w, (i + h * L) * kRun, dim, v[h]);
    }
}

template <class T, int L, int H>
__device__ __forceinline__ void load_row(const void *p, int64_t at, int i, int runs, int dim, float (&v)[H][kRun]) {
#pragma unroll
    for (int h = 0; h < H; h++) {
#pragma unroll
        for (int k = 0; k < kRun; k++) v[h][k] = 0.0f;
        if (i + h * L < runs) load_columns<T, kRun>(static_cast<const T *>(p) + at, (i + h * L) * kRun, dim, v[h]);
    }
}

template <class T, int L, int H, int kThreads>
__global__ __launch_bounds__(kThreads) void norm_kernel(const NormArgs a) {
    __shared__ double lds[2][kThreads / kWave][1];
    const int i = threadIdx.x % L;
    const int runs = (a.dim + kRun - 1) / kRun;
    float w[H][kRun], b[H][kRun];
    load_weights<L, H>(a.w, i, runs, a.dim, 1.0f, w);
    load_weights<L, H>(a.b, i, runs, a.dim, 0.0f, b);
    constexpr int kRows = kThreads / L;
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * kRows; at < a.n; at += static_cast<int64_t>(gridDim.x) * kRows) {
        const bool there = at + threadIdx.x / L < a.n;
        const int64_t row = there ? at + threadIdx.x / L : a.n - 1;
        float v[H][kRun];
        load_row<T, L, H>(a.x, row * a.xs, i, runs, a.dim, v);
        if (a.r) {
            float r[H][kRun];
            load_row<T, L, H>(a.r, row * a.rs, i, runs, a.dim, r);
#pragma unroll
            for (int h = 0; h < H; h++) {
#pragma unroll
                for (int k = 0; k < kRun; k++) v[h][k] = as_float(from_float<T>(v[h][k] + r[h][k]));
                if (there && i + h * L < runs)
                    store_columns<T, kRun>(static_cast<T *>(a.sum) + row * a.ss, (i + h * L) * kRun, a.dim, v[h]);
            }
        }
        double sum[1] = {0.0};
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < kRun; k++) sum[0] += v[h][k];       // 0 beyond the row
        row_sum<L>(sum, lds[0]);
        const double mean = sum[0] / a.dim;
        double squares[1] = {0.0};
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < kRun; k++) {
                const double c = (i + h * L) * kRun + k < a.dim ? v[h][k] - mean : 0.0;
                squares[0] = __builtin_fma(c, c, squares[0]);
            }
        row_sum<L>(squares, lds[1]);
        const double rstd = 1.0 / sqrt(squares[0] / a.dim + a.eps);
        if (!there) continue;
#pragma unroll
        for (int h = 0; h < H; h++) {
            if (i + h * L < runs) {
#pragma unroll
                for (int k = 0; k < kRun; k++)
                    v[h][k] = __builtin_fmaf(static_cast<float>((v[h][k] - mean) * rstd), w[h][k], b[h][k]);
                store_columns<T, kRun>(static_cast<T *>(a.y) + row * a.ys, (i + h * L) * kRun, a.dim, v[h]);
            }
        }
        if (a.stats && i == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = rstd;
        }
    }
}

template <class T, int L, int H, int kThreads, bool kParams>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(const GradArgs a) {
    __shared__ double lds[2][kThreads / kWave][2];
    const int i = threadIdx.x % L;
    const int runs = (a.dim + kRun - 1) / kRun;
    float w[H][kRun];
    load_weights<L, H>(a.w, i, runs, a.dim, 1.0f, w);
    double dw[kParams ? H : 1][kRun], db[kParams ? H : 1][kRun];
    if constexpr (kParams) {
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < kRun; k++) dw[h][k] = db[h][k] = 0.0;
    }
    constexpr int kRows = kThreads / L;
    int turn = 0;
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * kRows; at < a.n; at += static_cast<int64_t>(gridDim.x) * kRows) {
        const bool there = at + threadIdx.x / L < a.n;
        const int64_t row = there ? at + threadIdx.x / L : a.n - 1;
        float xh[H][kRun], dy[H][kRun];
        load_row<T, L, H>(a.h, row * a.hs, i, runs, a.dim, xh);
        load_row<T, L, H>(a.dy, row * a.dys, i, runs, a.dim, dy);
        const double mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        double sums[2] = {0.0, 0.0};
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < kRun; k++) {
                xh[h][k] = static_cast<float>((xh[h][k] - mean) * rstd);
                const double d = dy[h][k], g = d * w[h][k];             // 0 beyond the row
                if ((i + h * L) * kRun + k < a.dim) {
                    sums[0] += g;
                    sums[1] = __builtin_fma(g, static_cast<double>(xh[h][k]), sums[1]);
                    if constexpr (kParams) {
                        if (there) {
                            dw[h][k] = __builtin_fma(d, static_cast<double>(xh[h][k]), dw[h][k]);
                            db[h][k] += d;
                        }
                    }
                }
            }
        if (!a.dx) continue;
        row_sum<L>(sums, lds[turn]);
        turn ^= 1;
        if (!there) continue;
        const double c1 = sums[0] / a.dim, c2 = sums[1] / a.dim;
        float dh[H][kRun];
        if (a.dh) load_row<T, L, H>(a.dh, row * a.dhs, i, runs, a.dim, dh);
#pragma unroll
        for (int h = 0; h < H; h++) {
            if (i + h * L < runs) {
#pragma unroll
                for (int k = 0; k < kRun; k++) {
                    const double g = static_cast<double>(dy[h][k]) * w[h][k];
                    const double d = __builtin_fma(-c2, static_cast<double>(xh[h][k]), g - c1) * rstd;
                    dy[h][k] = static_cast<float>(a.dh ? d + dh[h][k] : d);
                }
                store_columns<T, kRun>(static_cast<T *>(a.dx) + row * a.dxs, (i + h * L) * kRun, a.dim, dy[h]);
            }
        }
    }
    if constexpr (kParams) {
        // the workgroup's rows together: first those of a wavefront, then its wavefronts one after another
        __shared__ double cols[L >= kWave || kThreads > kWave ? 2 : 1][L * H * kRun > 2048 ? 1 : L * H * kRun];
        double *part = a.parts + static_cast<int64_t>(blockIdx.x) * 2 * a.dim;
#pragma unroll
        for (int d = L; d < kWave; d <<= 1)
#pragma unroll
            for (int h = 0; h < H; h++)
#pragma unroll
                for (int k = 0; k < kRun; k++) {
                    dw[h][k] += __shfl_xor(dw[h][k], d, kWave);
                    db[h][k] += __shfl_xor(db[h][k], d, kWave);
                }
        constexpr int kWavesOfRow = L > kWave ? L / kWave : 1;
        constexpr int kGroups = kThreads / kWave / kWavesOfRow;
        if constexpr (kGroups == 1) {
#pragma unroll
            for (int h = 0; h < H; h++)
#pragma unroll
                for (int k = 0; k < kRun; k++) {
                    const int c = (i + h * L) * kRun + k;
                    if (c < a.dim && threadIdx.x < L) {
                        part[c] = dw[h][k];
                        part[a.dim + c] = db[h][k];
                    }
                }
        } else {
            const int group = threadIdx.x / kWave / kWavesOfRow;
            const bool owner = L >= kWave || lane_id() < L;
            for (int g = 0; g < kGroups; g++) {
                __syncthreads();
                if (g == group && owner) {
#pragma unroll
                    for (int h = 0; h < H; h++)
#pragma unroll
                        for (int k = 0; k < kRun; k++) {
                            const int c = (h * kRun + k) * L + i;           // lanes beside each other
                            cols[0][c] = g == 0 ? dw[h][k] : cols[0][c] + dw[h][k];
                            cols[1][c] = g == 0 ? db[h][k] : cols[1][c] + db[h][k];
                        }
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.dim; c += kThreads) {
                const int run = c / kRun, h = run / L, at = (h * kRun + c % kRun) * L + run % L;
                part[c] = cols[0][at];
                part[a.dim + c] = cols[1][at];
            }
        }
    }
}

// The workgroups' sums together, in their order within 64 slices: 16 columns a workgroup.
__global__ __launch_bounds__(1024) void norm_join_kernel(const double *parts, int32_t count, int32_t dim, float *dw, float *db) {
    __shared__ double lds[16][16];
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + threadIdx.x % 16;
    const int slice = threadIdx.x / 16;
    double sum = 0.0;
    if (c < 2 * static_cast<int64_t>(dim))
        for (int p = slice; p < count; p += 64) sum += parts[static_cast<int64_t>(p) * 2 * dim + c];
    sum += __shfl_xor(sum, 16, kWave);
    sum += __shfl_xor(sum, 32, kWave);
    if (lane_id() < 16) lds[threadIdx.x / kWave][lane_id()] = sum;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= 2 * static_cast<int64_t>(dim)) return;
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < 16; w++) sum += lds[w][threadIdx.x];
    if (c < dim) {
        if (dw) dw[c] = static_cast<float>(sum);
    } else if (db) {
        db[c - dim] = static_cast<float>(sum);
    }
}

// Workgroups of a call at most: the weights are read once for each, and their
// gradients' sums written once.
constexpr int64_t kBlocks = 4096;
int64_t grad_blocks(int32_t dim) { return dim <= 1024 ? 1024 : dim <= 4096 ? 512 : 256; }

// f(lanes of a row, runs of a lane, threads of a workgroup) for a row's width.
template <bool kGrad, class F>
void with_shape(int32_t dim, const F &f) {
    if (dim <= 64) f(Const<8>(), Const<1>(), Const<256>());
    else if (dim <= 128) f(Const<16>(), Const<1>(), Const<256>());
    else if (dim <= 256) f(Const<32>(), Const<1>(), Const<256>());
    else if (dim <= 512) f(Const<64>(), Const<1>(), Const<256>());
    else if (dim <= 1024) f(Const<64>(), Const<2>(), Const<256>());
    else if (dim <= 2048) f(Const<256>(), Const<1>(), Const<256>());
    else if (dim <= 4096) f(Const<512>(), Const<1>(), Const<512>());
    else if (dim <= 8192) f(Const<1024>(), Const<1>(), Const<1024>());
    else f(Const<1024>(), Const<2>(), Const<1024>());
}

template <class T>
tgl_status launch_norm(const NormArgs &a, hipStream_t st) {
    with_shape<false>(a.dim, [&](auto L, auto H, auto N) {
        constexpr int kL = decltype(L)::value, kH = decltype(H)::value, kN = decltype(N)::value;
        const int64_t blocks = (a.n + kN / kL - 1) / (kN / kL);
        norm_kernel<T, kL, kH, kN><<<static_cast<unsigned>(blocks < kBlocks ? blocks : kBlocks), kN, 0, st>>>(a);
    });
    return launch_status();
}

template <class T, bool kParams>
int64_t launch_grad(const GradArgs &a, hipStream_t st) {
    int64_t count = 0;
    with_shape<true>(a.dim, [&](auto L, auto H, auto N) {
        constexpr int kL = decltype(L)::value, kH = decltype(H)::value, kN = decltype(N)::value;
        const int64_t most = grad_blocks(a.dim), blocks = (a.n + kN / kL - 1) / (kN / kL);
        count = blocks < most ? blocks : most;
        norm_grad_kernel<T, kL, kH, kN, kParams><<<static_cast<unsigned>(count), kN, 0, st>>>(a);
    });
    return count;
}

bool valid_rows(int64_t n, int32_t dim, int32_t dtype) {
    return n >= 0 && dim >= 1 && dim <= TGL_MAX_NORM_DIM && is_elem_type(dtype);
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_layer_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                          const float *weight, const float *bias, int64_t n, int32_t dim, int32_t dtype, float eps,
                          void *y, int64_t y_stride, void *sum, int64_t sum_stride, double *stats, void *stream) {
    if (!valid_rows(n, dim, dtype) || !(eps >= 0.0f)) return TGL_EINVAL;
    const size_t e = elem_size(dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(y, e) || !aligned(sum, e) || !aligned(weight, 4) ||
        !aligned(bias, 4) || !aligned(stats, 8))
        return TGL_EINVAL;
    if (n > 0 && (!x || !y || (residual != nullptr) != (sum != nullptr))) return TGL_EINVAL;
    if (n > 1 && (y_stride < dim || (sum && sum_stride < dim))) return TGL_EINVAL;
    if (n == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const NormArgs a{x, residual, weight, bias, y, sum, stats, x_stride, residual_stride, y_stride, sum_stride, n, dim, eps};
    return dtype == TGL_OUT_F32 ? launch_norm<float>(a, st) : launch_norm<bf16_t>(a, st);
}

size_t tgl_layer_norm_grad_workspace(int64_t n, int32_t dim) {
    if (n < 0 || dim < 1 || dim > TGL_MAX_NORM_DIM) return 0;
    const int64_t most = grad_blocks(dim);
    return align_up(static_cast<size_t>(n < most ? n : most) * 2 * dim * sizeof(double), 256);
}

tgl_status tgl_layer_norm_grad(const void *dy, int64_t dy_stride, const void *h, int64_t h_stride,
                               const double *stats, const float *weight, const void *dsum, int64_t dsum_stride,
                               int64_t n, int32_t dim, int32_t dtype, void *dx, int64_t dx_stride, float *dweight,
                               float *dbias, void *workspace, size_t workspace_bytes, void *stream) {
    if (!valid_rows(n, dim, dtype)) return TGL_EINVAL;
    const size_t e = elem_size(dtype);
    if (!aligned(dy, e) || !aligned(h, e) || !aligned(dsum, e) || !aligned(dx, e) || !aligned(weight, 4) ||
        !aligned(stats, 8) || !aligned(dweight, 4) || !aligned(dbias, 4))
        return TGL_EINVAL;
    if (n > 0 && (!dy || !h || !stats || (n > 1 && dx && dx_stride < dim))) return TGL_EINVAL;
    const bool params = dweight || dbias;
    if (params && n > 0) {
        if (!workspace || workspace_bytes < tgl_layer_norm_grad_workspace(n, dim)) return TGL_ENOSPACE;
        if (!aligned(workspace, 256)) return TGL_EINVAL;
    }
    if (!dx && !params) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const GradArgs a{dy, h, dsum, stats, weight, dx, static_cast<double *>(workspace),
                     dy_stride, h_stride, dsum_stride, dx_stride, n, dim};
    int64_t count = 0;
    if (n > 0) {
        if (dtype == TGL_OUT_F32) count = params ? launch_grad<float, true>(a, st) : launch_grad<float, false>(a, st);
        else count = params ? launch_grad<bf16_t, true>(a, st) : launch_grad<bf16_t, false>(a, st);
        if (launch_status() != TGL_OK) return TGL_EDEVICE;
    }
    if (params)
        norm_join_kernel<<<static_cast<unsigned>((2 * dim + 15) / 16), 1024, 0, st>>>(a.parts, static_cast<int32_t>(count), dim,
                                                                                   dweight, dbias);
    return launch_status();
}

}  // extern "C"
