// tgl_rows8.hip -- residual addition, root-mean-square norm and rounding of
// rows to 8 bits.
//
//   h = x + r;  t = h * w;  a = max |t|;  s = a * (1 / 127);  q = rint(t * (1 / s))
//   scale = s / sqrt(mean(h^2) + eps)
//
// The norm's factor 1 / sqrt(mean + eps) is common to a row, so it drops out
// of the bytes and enters the scale alone: bytes do not depend on the order in
// which the mean's sum is taken.  Squares are summed in 64 bits: float32 ones of
// finite rows leave the range above 2^63 and below 2^-63.
#include "tgl_int8.hpp"

namespace tgl {
namespace {

// Workgroups of a call at most: the weights are read once for each.
constexpr int64_t kBlocks = 4096;

struct NormArgs {
    const void *x;
    const void *r;
    const float *w;
    int8_t *q;
    float *scale;
    void *sum;
    int64_t xs, rs, qs, ss;
    int64_t n;
    int32_t dim;
    int32_t normalize;
    float eps;
};

constexpr int kRun = 8;             // elements of a lane's access

// step / sqrt(mean + eps), in float32 where that has the range.
__device__ __forceinline__ float normed_step(const NormArgs &a, float step, double squares) {
    if (!a.normalize) return step;
    const double x = squares / a.dim + a.eps;
    if (x > 0x1p-100 && x < 0x1p100) return step / sqrtf(static_cast<float>(x));
    return static_cast<float>(step / sqrt(x));
}

// L lanes per row, which stays in registers: H runs of 8 elements a lane.  The
// weights of a lane's columns stay there too, over all rows it takes.  Bound by
// memory: 12,000 rows of 768 bfloat16 with a residual (64 MB) 16.4 us, 3.9 TB/s
// (34 us in two passes over each row); one row 3.4 us, two latencies of memory
// and the exchanges of two sums.
template <class T, int L, int H>
__global__ __launch_bounds__(kBlock) void norm_kernel(const NormArgs a) {
    constexpr int kWaves = L / kWave;           // of a row
    __shared__ float tops[kBlock / kWave];
    __shared__ double parts[kBlock / kWave];
    const int i = threadIdx.x % L;
    const int group = threadIdx.x / L;
    const int runs = round16(a.dim) / kRun;
    float w[H][kRun];
#pragma unroll
    for (int h = 0; h < H; h++) {
        if (a.w && i + h * L < runs) load_columns<float, kRun>(a.w, (i + h * L) * kRun, a.dim, w[h]);
        else for (int k = 0; k < kRun; k++) w[h][k] = 1.0f;
    }
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (kBlock / L);
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * (kBlock / L); at < a.n; at += stride) {
        const bool there = at + group < a.n;
        const int64_t row = there ? at + group : a.n - 1;
        const T *x = static_cast<const T *>(a.x) + row * a.xs;
        const T *r = static_cast<const T *>(a.r) + row * a.rs;
        float v[H][kRun];
#pragma unroll
        for (int h = 0; h < H; h++) {
            if (i + h * L < runs) load_columns<T, kRun>(x, (i + h * L) * kRun, a.dim, v[h]);
            else for (int k = 0; k < kRun; k++) v[h][k] = 0.0f;
        }
        if (a.r) {
#pragma unroll
            for (int h = 0; h < H; h++) {
                if (i + h * L < runs) {
                    float y[kRun];
                    load_columns<T, kRun>(r, (i + h * L) * kRun, a.dim, y);
#pragma unroll
                    for (int k = 0; k < kRun; k++) v[h][k] += y[k];
                }
            }
        }
        double squares = 0.0;
        uint32_t bits = 0;              // of the largest magnitude: NaN above infinity above numbers
#pragma unroll
        for (int h = 0; h < H; h++) {
#pragma unroll
            for (int k = 0; k < kRun; k++) squares = __builtin_fma(static_cast<double>(v[h][k]), static_cast<double>(v[h][k]), squares);
            if (a.sum && there && i + h * L < runs)
                store_columns<T, kRun>(static_cast<T *>(a.sum) + row * a.ss, (i + h * L) * kRun, a.dim, v[h]);
#pragma unroll
            for (int k = 0; k < kRun; k++) {
                v[h][k] *= w[h][k];
                const uint32_t y = __builtin_bit_cast(uint32_t, v[h][k]) & 0x7fffffffu;
                bits = y > bits ? y : bits;
            }
        }
#pragma unroll
        for (int d = kWave / 2; d >= 1; d >>= 1) {
            squares += __shfl_xor(squares, d, kWave);
            const uint32_t y = __shfl_xor(bits, d, kWave);
            bits = y > bits ? y : bits;
        }
        if constexpr (kWaves > 1) {
            __syncthreads();            // the last row's readers are done
            if (lane_id() == 0) {
                tops[threadIdx.x / kWave] = __builtin_bit_cast(float, bits);
                parts[threadIdx.x / kWave] = squares;
            }
            __syncthreads();
            squares = 0.0;
#pragma unroll
            for (int y = 0; y < kWaves; y++) {
                squares += parts[group * kWaves + y];
                const uint32_t t = __builtin_bit_cast(uint32_t, tops[group * kWaves + y]);
                bits = t > bits ? t : bits;
            }
        }
        const float s = step_of(__builtin_bit_cast(float, bits)), inv = inverse_step(s);
        if (!there) continue;
#pragma unroll
        for (int h = 0; h < H; h++) {
            if (i + h * L < runs) {
                i32x2 q = {0, 0};
                if (inv != 0.0f)
                    q = i32x2{to_bytes4(v[h][0], v[h][1], v[h][2], v[h][3], inv), to_bytes4(v[h][4], v[h][5], v[h][6], v[h][7], inv)};
                *reinterpret_cast<i32x2 *>(a.q + row * a.qs + (i + h * L) * kRun) = q;
            }
        }
        if (i == 0) a.scale[row] = normed_step(a, s, squares);
    }
}

// Rows that no workgroup's registers hold (above 8192 elements), in two passes
// over each, the second mostly from L2.
template <class T>
__global__ __launch_bounds__(kBlock) void norm_long_kernel(const NormArgs a) {
    __shared__ float tops[kBlock / kWave];
    __shared__ double parts[kBlock / kWave];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.xs;
        const T *r = a.r ? static_cast<const T *>(a.r) + row * a.rs : nullptr;
        double squares = 0.0;
        uint32_t bits = 0;
        auto hold = [&](int n, float (&h)[kRun], float (&t)[kRun]) {
            load_columns<T, kRun>(x, n * kRun, a.dim, h);
            if (r) {
                load_columns<T, kRun>(r, n * kRun, a.dim, t);
#pragma unroll
                for (int k = 0; k < kRun; k++) h[k] += t[k];
            }
#pragma unroll
            for (int k = 0; k < kRun; k++) t[k] = 1.0f;
            if (a.w) load_columns<float, kRun>(a.w, n * kRun, a.dim, t);
#pragma unroll
            for (int k = 0; k < kRun; k++) t[k] *= h[k];
        };
        const int runs = round16(a.dim) / kRun;
        for (int n = threadIdx.x; n < runs; n += kBlock) {
            float h[kRun], t[kRun];
            hold(n, h, t);
#pragma unroll
            for (int k = 0; k < kRun; k++) {
                squares = __builtin_fma(static_cast<double>(h[k]), static_cast<double>(h[k]), squares);
                const uint32_t y = __builtin_bit_cast(uint32_t, t[k]) & 0x7fffffffu;
                bits = y > bits ? y : bits;
            }
        }
#pragma unroll
        for (int d = kWave / 2; d >= 1; d >>= 1) {
            squares += __shfl_xor(squares, d, kWave);
            const uint32_t y = __shfl_xor(bits, d, kWave);
            bits = y > bits ? y : bits;
        }
        __syncthreads();
        if (lane_id() == 0) {
            tops[threadIdx.x / kWave] = __builtin_bit_cast(float, bits);
            parts[threadIdx.x / kWave] = squares;
        }
        __syncthreads();
        squares = 0.0;
#pragma unroll
        for (int y = 0; y < kBlock / kWave; y++) {
            squares += parts[y];
            const uint32_t t = __builtin_bit_cast(uint32_t, tops[y]);
            bits = t > bits ? t : bits;
        }
        const float s = step_of(__builtin_bit_cast(float, bits)), inv = inverse_step(s);
        for (int n = threadIdx.x; n < runs; n += kBlock) {
            float h[kRun], t[kRun];
            hold(n, h, t);
            i32x2 q = {0, 0};
            if (inv != 0.0f) q = i32x2{to_bytes4(t[0], t[1], t[2], t[3], inv), to_bytes4(t[4], t[5], t[6], t[7], inv)};
            *reinterpret_cast<i32x2 *>(a.q + row * a.qs + n * kRun) = q;
            if (a.sum) store_columns<T, kRun>(static_cast<T *>(a.sum) + row * a.ss, n * kRun, a.dim, h);
        }
        if (threadIdx.x == 0) a.scale[row] = normed_step(a, s, squares);
    }
}

template <class T, int L, int H>
void launch_norm(const NormArgs &a, hipStream_t st) {
    constexpr int64_t kRowsOf = kBlock / L;
    const int64_t blocks = (a.n + kRowsOf - 1) / kRowsOf;
    norm_kernel<T, L, H><<<static_cast<unsigned>(blocks < kBlocks ? blocks : kBlocks), kBlock, 0, st>>>(a);
}

template <class T>
void launch_norm(const NormArgs &a, hipStream_t st) {
    const int runs = round16(a.dim) / kRun;
    if (runs <= 64) launch_norm<T, 64, 1>(a, st);
    else if (runs <= 128) launch_norm<T, 64, 2>(a, st);
    else if (runs <= 256) launch_norm<T, 256, 1>(a, st);
    else if (runs <= 512) launch_norm<T, 256, 2>(a, st);
    else if (runs <= 1024) launch_norm<T, 256, 4>(a, st);
    else norm_long_kernel<T><<<static_cast<unsigned>(a.n < kBlocks ? a.n : kBlocks), kBlock, 0, st>>>(a);
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_norm_quant(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                          const float *weight, int64_t n, int32_t dim, int32_t dtype, int32_t normalize,
                          float eps, int8_t *q, int64_t q_stride, float *scale, void *sum,
                          int64_t sum_stride, void *stream) {
    if (n < 0 || dim < 1 || dim > TGL_MAX_ROW_DIM || !is_elem_type(dtype) || (normalize != 0 && normalize != 1))
        return TGL_EINVAL;
    if (normalize && !(eps >= 0.0f)) return TGL_EINVAL;
    const size_t e = elem_size(dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(sum, e) || !aligned(weight, 4) || !aligned(scale, 4))
        return TGL_EINVAL;
    if (!aligned(q, 16) || q_stride % 16 != 0 || q_stride < dim) return TGL_EINVAL;
    if (sum && sum_stride < dim) return TGL_EINVAL;
    if (n > 0 && (!x || !q || !scale)) return TGL_EINVAL;
    if (n == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const NormArgs a{x, residual, weight, q, scale, sum, x_stride, residual_stride, q_stride, sum_stride, n, dim, normalize, eps};
    if (dtype == TGL_OUT_F32) launch_norm<float>(a, st);
    else launch_norm<bf16_t>(a, st);
    return launch_status();
}

}  // extern "C"
