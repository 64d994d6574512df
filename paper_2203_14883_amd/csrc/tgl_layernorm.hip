// tgl_layernorm.hip -- residual addition and layer norm of rows, and their
// gradients.
//
//   h = x + r;  m = mean(h);  s = 1 / sqrt(mean((h - m)^2) + eps);  y = (h - m) s w + b
//   xh = (h - m) s;  g = dy w;  dx = (g - mean(g) - xh mean(g xh)) s + dh
//   dw = sum dy xh;  db = sum dy
//
// A row is read once and stays in the registers of L lanes, so the mean of the
// squared distances is taken from the distances themselves.  The norm's sums, and
// distances before they are scaled, are of 64 bits: squares of finite float32
// numbers leave that type's range, and a mean that is large beside the
// distances would lose their bits in 32.  The card does 64-bit sums and
// products at the rate of float32's, and memory bounds these kernels.  What the
// gradients sum in 32 bits first is said there.
#include <type_traits>

#include "tgl_typed.hpp"

namespace tgl {
namespace {

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

// What the lane whose number differs in bit D has (for D = 4 and 8: one of the
// other half's, which all have the same by then).  In registers: exchanges through LDS
// would be most of a row's time.
template <int D>
__device__ __forceinline__ double exchanged(double v) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    uint32_t half[2] = {static_cast<uint32_t>(bits), static_cast<uint32_t>(bits >> 32)};
#pragma unroll
    for (int i = 0; i < 2; i++) {
        if constexpr (D < 16) {
            constexpr int kControl = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 4 ? 0x141 : 0x140;   // quads, half rows, rows of 16
            half[i] = __builtin_amdgcn_update_dpp(0, half[i], kControl, 0xf, 0xf, true);
        } else {
            const auto both = D == 16 ? __builtin_amdgcn_permlane16_swap(half[i], half[i], false, false)
                                      : __builtin_amdgcn_permlane32_swap(half[i], half[i], false, false);
            half[i] = lane_id() & D ? both[0] : both[1];
        }
    }
    return __builtin_bit_cast(double, static_cast<uint64_t>(half[1]) << 32 | half[0]);
}

// Sum over the L lanes of a row, in all of them.  `lds` has one number per wavefront of
// the workgroup and is free again after the next barrier.
template <int L, int N>
__device__ __forceinline__ void row_sum(double (&v)[N], double (*lds)[N]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        v[i] += exchanged<1>(v[i]);
        v[i] += exchanged<2>(v[i]);
        v[i] += exchanged<4>(v[i]);
        if constexpr (L >= 16) v[i] += exchanged<8>(v[i]);
        if constexpr (L >= 32) v[i] += exchanged<16>(v[i]);
        if constexpr (L >= 64) v[i] += exchanged<32>(v[i]);
    }
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

constexpr int E = 4;                // elements of a run, a lane's access

// A run as whole words, which are taken apart where its elements are used: so nothing waits for a load before that.
template <class T>
using run_t = std::conditional_t<sizeof(T) == 2, i32x2, i32x4>;

template <class T>
__device__ __forceinline__ float run_at(const run_t<T> &v, int k) {
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, k & 1 ? v[k / 2] & static_cast<int>(0xffff0000u) : v[k / 2] << 16);
    else return __builtin_bit_cast(f32x4, v)[k];
}

// Run h of lane i of a row's L begins at column (i + h L) E.  Zeros beyond the
// row; kWhole: rows end with a run.
template <class T, int L, bool kWhole>
__device__ __forceinline__ run_t<T> load_run(const void *p, int64_t at, int i, int h, int dim) {
    using word_t = run_t<T> __attribute__((aligned(alignof(T))));
    const T *row = static_cast<const T *>(p) + at;
    const int c = (i + h * L) * E;
    if constexpr (kWhole) {
        run_t<T> v = {};
        if (c < dim) v = *reinterpret_cast<const word_t *>(row + c);
        return v;
    }
    if (c + E <= dim) return *reinterpret_cast<const word_t *>(row + c);
    Run<T, E> v = {};
#pragma unroll
    for (int k = 0; k < E; k++)
        if (c + k < dim) v.t[k] = row[c + k];
    return __builtin_bit_cast(run_t<T>, v);
}

// A row in the registers of L lanes.
template <class T, int L, int H, bool kWhole>
struct Held {
    run_t<T> v[H];
    __device__ __forceinline__ void load(const void *p, int64_t at, int i, int dim) {
#pragma unroll
        for (int h = 0; h < H; h++) v[h] = load_run<T, L, kWhole>(p, at, i, h, dim);
    }
    __device__ __forceinline__ float at(int h, int k) const { return run_at<T>(v[h], k); }
};

// E columns from c < dim on.
template <class T, bool kWhole>
__device__ __forceinline__ void store_run(void *p, int64_t at, int c, int dim, const float (&v)[E]) {
    store_columns<T, E>(static_cast<T *>(p) + at, c, kWhole ? c + E : dim, v);
}

template <class T, int L, int H, bool kWhole>
__device__ __forceinline__ void store_row(void *p, int64_t at, int i, int dim, const float (&v)[H][E]) {
#pragma unroll
    for (int h = 0; h < H; h++)
        if ((i + h * L) * E < dim) store_run<T, kWhole>(p, at, (i + h * L) * E, dim, v[h]);
}

// A lane's columns of the weights, or what stands for none.
template <class T, int L, int H>
__device__ __forceinline__ void load_weights(const float *w, int i, int dim, float without, float (&v)[H][E]) {
#pragma unroll
    for (int h = 0; h < H; h++) {
#pragma unroll
        for (int k = 0; k < E; k++) v[h][k] = without;
        if (w && (i + h * L) * E < dim) load_columns<float, E>(w, (i + h * L) * E, dim, v[h]);
    }
}

// Bound by memory, as long as enough of it is on its way: the next row is loaded
// before this one is worked on, where registers have room (kAhead).
template <class T, int L, int H, int kThreads, bool kAhead, bool kWhole>
__global__ __launch_bounds__(kThreads) void norm_kernel(const NormArgs a) {
    __shared__ double lds[2][kThreads / kWave][1];
    constexpr int kRows = kThreads / L;
    const int i = threadIdx.x % L, sub = threadIdx.x / L;
    float w[H][E], b[H][E];
    load_weights<T, L, H>(a.w, i, a.dim, 1.0f, w);
    load_weights<T, L, H>(a.b, i, a.dim, 0.0f, b);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kRows;
    auto row_of = [&](int64_t at) { return at + sub < a.n ? at + sub : a.n - 1; };
    Held<T, L, H, kWhole> x, r, next_x, next_r;
    auto load = [&](int64_t at, auto &x, auto &r) {
        x.load(a.x, row_of(at) * a.xs, i, a.dim);
        if (a.r) r.load(a.r, row_of(at) * a.rs, i, a.dim);
    };
    int64_t at = static_cast<int64_t>(blockIdx.x) * kRows;
    load(at, x, r);
    for (; at < a.n; at += stride) {
        if (kAhead && at + stride < a.n) load(at + stride, next_x, next_r);
        const bool there = at + sub < a.n;
        const int64_t row = row_of(at);
        float v[H][E];
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < E; k++) {
                v[h][k] = x.at(h, k);
                if (a.r) v[h][k] = as_float(from_float<T>(v[h][k] + r.at(h, k)));
            }
        if (a.r && there) store_row<T, L, H, kWhole>(a.sum, row * a.ss, i, a.dim, v);
        double sum[1] = {0.0};
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < E; k++) sum[0] += v[h][k];
        row_sum<L>(sum, lds[0]);
        const double mean = sum[0] / a.dim;
        double squares[1] = {0.0};
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < E; k++) {
                const double c = (i + h * L) * E + (kWhole ? 0 : k) < a.dim ? v[h][k] - mean : 0.0;
                squares[0] = __builtin_fma(c, c, squares[0]);
            }
        row_sum<L>(squares, lds[1]);
        const double rstd = 1.0 / sqrt(squares[0] / a.dim + a.eps);
        if (there) {
#pragma unroll
            for (int h = 0; h < H; h++)
#pragma unroll
                for (int k = 0; k < E; k++)
                    v[h][k] = __builtin_fmaf(static_cast<float>((v[h][k] - mean) * rstd), w[h][k], b[h][k]);
            store_row<T, L, H, kWhole>(a.y, row * a.ys, i, a.dim, v);
            if (a.stats && i == 0) {
                a.stats[2 * row] = mean;
                a.stats[2 * row + 1] = rstd;
            }
        }
        if constexpr (kAhead) {
            x = next_x;
            r = next_r;
        } else {
            if (at + stride < a.n) load(at + stride, x, r);
        }
    }
}

constexpr float kMost = 3.4028235e38f;      // of float32

// All loads are done.  Said where the next row takes this one's place: left to the compiler, the wait may come where that row is
// first used, behind the loads of the one after it, and wait for those too (30,000 rows of 2048 bfloat16 131 us, 110 so).
__device__ __forceinline__ void arrived() { __builtin_amdgcn_s_waitcnt(0x0f70); }       // vmcnt(0)

// Rows of a lane whose products are summed in 32 bits before they join its 64-bit sums.
constexpr int kChain = 32;

// As norm_kernel, but 64-bit numbers for all of it would take more than memory
// does (52 operations an element, 280 us for 132,000 rows of 768 bfloat16 with a sum's
// gradient, where these take 18): distances from the mean are taken from its upper and
// its lower bits, (h - upper) - lower, which loses nothing that 32 bits could hold, and a row's
// means and the weights' gradients are sums of 64 bits of a lane's few elements, or kChain rows,
// in 32.  Rows that leave float32's range on the way (in their mean, 1 / sigma, products or sums)
// are worked in 64; the weights' sums of kChain rows have float32's range.  Rows too
// wide for the registers (!kHold) are read again, mostly from L2, once their means are known.
template <class T, int L, int H, int kThreads, bool kHold, bool kWhole, bool kParams>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(const GradArgs a) {
    __shared__ double lds[2][kThreads / kWave][2];
    constexpr int kRows = kThreads / L, kColumns = L * H * E;
    constexpr int kWavesOfRow = L > kWave ? L / kWave : 1, kGroups = kThreads / kWave / kWavesOfRow;
    __shared__ double cols[2][kParams && kGroups > 1 ? kColumns : 1];
    const int i = threadIdx.x % L, sub = threadIdx.x / L;
    float w[H][E];
    load_weights<T, L, H>(a.w, i, a.dim, 1.0f, w);
    float dw[kParams ? H : 1][E] = {}, db[kParams ? H : 1][E] = {};
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kRows;

    Held<T, L, kHold ? H : 1, kWhole> dy, x, dh, next_dy, next_x, next_dh;
    double mean, rstd, next_mean = 0.0, next_rstd = 0.0;
    // rows beyond the last are zeros
    auto load = [&](int64_t at, auto &dy, auto &x, auto &dh, double &mean, double &rstd) {
        const bool there = at + sub < a.n;
        const int64_t row = there ? at + sub : a.n - 1;
        if constexpr (kHold) {
            const int dim = there ? a.dim : 0;
            dy.load(a.dy, row * a.dys, i, dim);
            x.load(a.h, row * a.hs, i, dim);
            if (a.dh) dh.load(a.dh, row * a.dhs, i, dim);
        }
        mean = there ? a.stats[2 * row] : 0.0;
        rstd = there ? a.stats[2 * row + 1] : 0.0;
    };
    // The lanes' sums of the weights' gradients to the workgroup's: first those of a
    // wavefront, then its wavefronts one after another.
    auto flush = [&](bool first) {
        double *part = a.parts + static_cast<int64_t>(blockIdx.x) * 2 * a.dim;
        auto add = [&](int c, double x, double y) {
            part[c] = first ? x : part[c] + x;
            part[a.dim + c] = first ? y : part[a.dim + c] + y;
        };
        if constexpr (kGroups == 1) {
#pragma unroll
            for (int h = 0; h < H; h++)
#pragma unroll
                for (int k = 0; k < E; k++)
                    if ((i + h * L) * E + k < a.dim) add((i + h * L) * E + k, dw[h][k], db[h][k]);
        } else {
            const int group = threadIdx.x / kWave / kWavesOfRow;
            const bool owner = L >= kWave || lane_id() < L;
            for (int g = 0; g < kGroups; g++) {
                __syncthreads();
                if (g != group) continue;
#pragma unroll
                for (int h = 0; h < H; h++)
#pragma unroll
                    for (int k = 0; k < E; k++) {
                        double x = dw[h][k], y = db[h][k];
#pragma unroll
                        for (int d = L; d < kWave; d <<= 1) {
                            x += __shfl_xor(x, d, kWave);
                            y += __shfl_xor(y, d, kWave);
                        }
                        const int c = (h * E + k) * L + i;                  // lanes beside each other
                        if (owner) {
                            cols[0][c] = g == 0 ? x : cols[0][c] + x;
                            cols[1][c] = g == 0 ? y : cols[1][c] + y;
                        }
                    }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.dim; c += kThreads) {
                const int run = c / E, at = (run / L * E + c % E) * L + run % L;
                add(c, cols[0][at], cols[1][at]);
            }
        }
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int k = 0; k < E; k++) dw[h][k] = db[h][k] = 0.0f;
    };
    int64_t at = static_cast<int64_t>(blockIdx.x) * kRows;
    load(at, dy, x, dh, mean, rstd);
    arrived();
    int turn = 0, rows = 0;
    bool flushed = false;
    for (; at < a.n; at += stride) {
        if (at + stride < a.n) load(at + stride, next_dy, next_x, next_dh, next_mean, next_rstd);
        const bool there = at + sub < a.n;
        const int64_t row = there ? at + sub : a.n - 1;
        const int dim = there ? a.dim : 0;
        // mean rstd is what normed() gives for the zeros beyond the row, where g is 0: their product has to be a number
        const bool ordinary = fabs(mean) < 0x1p100 && rstd > 0x1p-60 && rstd < 0x1p60 && fabs(mean) * rstd < 0x1p100;
        const float upper = static_cast<float>(mean), lower = static_cast<float>(mean - upper), scale = static_cast<float>(rstd);
        auto run_of = [&](const auto &held, const void *p, int64_t stride, int h) {
            if constexpr (kHold) return held.v[h];
            else return load_run<T, L, kWhole>(p, row * stride, i, h, dim);
        };
        auto normed = [&](float v) { return ((v - upper) - lower) * scale; };
        // beyond the row 0, as dy is there: the product need not be a number
        auto normed_wide = [&](float v, int c) { return c < dim ? static_cast<float>((v - mean) * rstd) : 0.0f; };
        // A run once more from memory, where float32 is left: held in registers for that, rows would take more of them than all
        // else does.  opaque: addresses are not worked out, and kept, for rows that need none.
        auto again = [&](int64_t row, int i, int h, run_t<T> &dv, run_t<T> &xv, float(&wv)[E]) {
            dv = load_run<T, L, kWhole>(a.dy, row * a.dys, i, h, dim);
            xv = load_run<T, L, kWhole>(a.h, row * a.hs, i, h, dim);
#pragma unroll
            for (int k = 0; k < E; k++) wv[k] = 1.0f;
            if (a.w && (i + h * L) * E < a.dim) load_columns<float, E>(a.w, (i + h * L) * E, a.dim, wv);
        };
        auto opaque = [](auto v) {
            asm volatile("" : "+v"(v));
            return v;
        };
        float xh[kHold ? H : 1][E];
        float part[2] = {0.0f, 0.0f};
#pragma unroll
        for (int h = 0; h < H; h++) {
            const run_t<T> dv = run_of(dy, a.dy, a.dys, h), xv = run_of(x, a.h, a.hs, h);
            float t[E];
            if (ordinary) {
#pragma unroll
                for (int k = 0; k < E; k++) t[k] = normed(run_at<T>(xv, k));
            } else {
#pragma unroll
                for (int k = 0; k < E; k++) t[k] = normed_wide(run_at<T>(xv, k), (i + h * L) * E + k);
            }
#pragma unroll
            for (int k = 0; k < E; k++) {
                const float d = run_at<T>(dv, k), g = d * w[h][k];
                part[0] += g;
                part[1] = __builtin_fmaf(g, t[k], part[1]);
                if constexpr (kParams) {
                    dw[h][k] = __builtin_fmaf(d, t[k], dw[h][k]);
                    db[h][k] += d;
                }
                if constexpr (kHold) xh[h][k] = t[k];
            }
        }
        if (a.dx) {
            double sums[2] = {part[0], part[1]};
            // a product of the lane, or a sum, is beyond float32 (once it is, the sum is no finite number again)
            const bool large = !(fabsf(part[0]) + fabsf(part[1]) <= kMost);
            if (__builtin_expect(large, false)) {
                sums[0] = sums[1] = 0.0;
#pragma unroll 1
                for (int h = 0; h < H; h++) {
                    run_t<T> dv, xv;
                    float wv[E];
                    const int lane = opaque(i);
                    again(opaque(row), lane, h, dv, xv, wv);
#pragma unroll
                    for (int k = 0; k < E; k++) {
                        const double g = static_cast<double>(run_at<T>(dv, k)) * wv[k];
                        sums[0] += g;
                        sums[1] = __builtin_fma(g, static_cast<double>(normed_wide(run_at<T>(xv, k), (lane + h * L) * E + k)), sums[1]);
                    }
                }
            }
            row_sum<L>(sums, lds[turn]);
            turn ^= 1;
            const double inv = 1.0 / a.dim, c1 = sums[0] * inv, c2 = sums[1] * inv;
            const float c1f = static_cast<float>(c1), c2f = static_cast<float>(c2);
            // then nothing on the way leaves float32: what is subtracted, of |xh| below 2^8, is less than half a unit of its largest number
            const bool within = ordinary && !large && fmaxf(fabsf(c1f), fabsf(c2f)) < 0x1p90f;
            if (__builtin_expect(there && within, true)) {
#pragma unroll
                for (int h = 0; h < H; h++) {
                    const int c = (i + h * L) * E;
                    if (c >= a.dim) continue;
                    const run_t<T> dv = run_of(dy, a.dy, a.dys, h);
                    run_t<T> xv = {}, hv = {};
                    if constexpr (!kHold) xv = run_of(x, a.h, a.hs, h);
                    if (a.dh) hv = run_of(dh, a.dh, a.dhs, h);
                    float v[E];
#pragma unroll
                    for (int k = 0; k < E; k++) {
                        const float t = kHold ? xh[kHold ? h : 0][k] : normed(run_at<T>(xv, k));
                        v[k] = __builtin_fmaf(-c2f, t, run_at<T>(dv, k) * w[h][k] - c1f);
                        v[k] = __builtin_fmaf(v[k], scale, run_at<T>(hv, k));
                    }
                    store_run<T, kWhole>(a.dx, row * a.dxs, c, a.dim, v);
                }
            } else if (there) {
#pragma unroll 1
                for (int h = 0; h < H; h++) {
                    const int lane = opaque(i), c = (lane + h * L) * E;
                    const int64_t own = opaque(row);
                    if (c >= a.dim) break;
                    run_t<T> dv, xv, hv = {};
                    float wv[E], v[E];
                    again(own, lane, h, dv, xv, wv);
                    if (a.dh) hv = load_run<T, L, kWhole>(a.dh, own * a.dhs, lane, h, dim);
#pragma unroll
                    for (int k = 0; k < E; k++) {
                        const double t = normed_wide(run_at<T>(xv, k), c + k);
                        const double d = __builtin_fma(-c2, t, static_cast<double>(run_at<T>(dv, k)) * wv[k] - c1) * rstd;
                        v[k] = static_cast<float>(d + run_at<T>(hv, k));
                    }
                    store_run<T, kWhole>(a.dx, own * a.dxs, c, a.dim, v);
                }
            }
        }
        if constexpr (kParams) {
            if (++rows == kChain) {
                flush(!flushed);
                flushed = true;
                rows = 0;
            }
        }
        arrived();
        if constexpr (kHold) {
            dy = next_dy;
            x = next_x;
            dh = next_dh;
        }
        mean = next_mean;
        rstd = next_rstd;
    }
    if constexpr (kParams) {
        if (rows || !flushed) flush(!flushed);
    }
}

// The workgroups' sums together, in their order within 64 slices: 16 columns a workgroup.
__global__ __launch_bounds__(1024) void norm_join_kernel(const double *parts, int32_t count, int32_t dim, float *dw, float *db) {
    __shared__ double lds[16][16];
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + threadIdx.x % 16;
    const int slice = threadIdx.x / 16;
    double sum = 0.0;
    if (c < 2 * static_cast<int64_t>(dim)) {
#pragma unroll 8
        for (int p = slice; p < count; p += 64) sum += parts[static_cast<int64_t>(p) * 2 * dim + c];
    }
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

// Workgroups of a call at most: each takes several rows in turn, four where there
// are enough for every compute unit, and reads the weights and writes the sums of their gradients once.
constexpr int64_t kBlocks = 2048;
// Rows of three runs a lane: two wavefronts a SIMD (132,000 x 768 bfloat16 156 us), not the three that fit (168).
int64_t grad_blocks(int32_t dim) { return dim <= 512 ? 1024 : dim <= 768 ? 512 : dim <= 1024 ? 1024 : dim <= 4096 ? 512 : 256; }

// f(lanes of a row, runs of a lane, threads of a workgroup, whether a row stays in registers) for a row's width.
template <class F>
void with_shape(int32_t dim, const F &f) {
    using Yes = std::true_type;
    using No = std::false_type;
    if (dim <= 32) f(Const<8>(), Const<1>(), Const<256>(), Yes());
    else if (dim <= 64) f(Const<16>(), Const<1>(), Const<256>(), Yes());
    else if (dim <= 128) f(Const<32>(), Const<1>(), Const<256>(), Yes());
    else if (dim <= 256) f(Const<64>(), Const<1>(), Const<256>(), Yes());
    else if (dim <= 512) f(Const<64>(), Const<2>(), Const<256>(), Yes());
    else if (dim <= 768) f(Const<64>(), Const<3>(), Const<256>(), Yes());
    else if (dim <= 1024) f(Const<128>(), Const<2>(), Const<256>(), Yes());
    else if (dim <= 2048) f(Const<256>(), Const<2>(), Const<256>(), Yes());
    else if (dim <= 4096) f(Const<512>(), Const<2>(), Const<512>(), Yes());
    else if (dim <= 8192) f(Const<512>(), Const<4>(), Const<512>(), No());
    else f(Const<512>(), Const<8>(), Const<512>(), No());
}

template <class T>
tgl_status launch_norm(const NormArgs &a, hipStream_t st) {
    with_shape(a.dim, [&](auto L, auto H, auto N, auto Hold) {
        constexpr int kL = decltype(L)::value, kH = decltype(H)::value, kN = decltype(N)::value;
        const int64_t blocks = (a.n + kN / kL - 1) / (kN / kL);
        const unsigned grid = static_cast<unsigned>(blocks < kBlocks ? blocks : kBlocks);
        if (a.dim % E == 0) norm_kernel<T, kL, kH, kN, decltype(Hold)::value, true><<<grid, kN, 0, st>>>(a);
        else norm_kernel<T, kL, kH, kN, decltype(Hold)::value, false><<<grid, kN, 0, st>>>(a);
    });
    return launch_status();
}

// Workgroups that the card holds at a time: all rows are shared among these, and no few workgroups come after them
// (for float32 1024, where it holds 768: 132,000 rows of 300 151 us, 126 so; 40,000 of 1024 144 and 130).
template <class K>
int resident_blocks(K kernel, int threads) {
    int each = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, threads, 0) != hipSuccess || each < 1) {
        (void)hipGetLastError();
        each = 1;
    }
    return each * 256;
}

template <class T, bool kParams>
int64_t launch_grad(const GradArgs &a, hipStream_t st) {
    int64_t count = 0;
    with_shape(a.dim, [&](auto L, auto H, auto N, auto Hold) {
        constexpr int kL = decltype(L)::value, kH = decltype(H)::value, kN = decltype(N)::value;
        const auto kernel = a.dim % E == 0 ? norm_grad_kernel<T, kL, kH, kN, decltype(Hold)::value, true, kParams>
                                           : norm_grad_kernel<T, kL, kH, kN, decltype(Hold)::value, false, kParams>;
        static const int resident[2] = {resident_blocks(norm_grad_kernel<T, kL, kH, kN, decltype(Hold)::value, true, kParams>, kN),
                                        resident_blocks(norm_grad_kernel<T, kL, kH, kN, decltype(Hold)::value, false, kParams>, kN)};
        int64_t most = grad_blocks(a.dim);
        if (most > resident[a.dim % E != 0]) most = resident[a.dim % E != 0];
        const int64_t blocks = (a.n + kN / kL - 1) / (kN / kL);
        count = blocks < 256 ? blocks : blocks / 4 < 256 ? 256 : blocks / 4 < most ? blocks / 4 : most;
        kernel<<<static_cast<unsigned>(count), kN, 0, st>>>(a);
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
