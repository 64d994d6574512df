// tgl_rows8.hip -- residual addition, root-mean-square norm and rounding of
// rows to 8 bits.
//
//   h = x + r;  t = h * w;  a = max |t|;  s = a * (1 / 127);  q = rint(t * (1 / s))
//   scale = s / sqrt(mean(h^2) + eps)
//
// The norm's factor 1 / sqrt(mean + eps) is common to a row, so it drops out
// of the bytes and enters the scale alone: bytes do not depend on the order in
// which the mean's sum is taken.
#include "tgl_int8.hpp"

namespace tgl {
namespace {

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

// A wavefront per row, in two passes over it.
template <class T>
__global__ __launch_bounds__(kBlock) void norm_kernel(const NormArgs a) {
    const int lane = lane_id();
    const int64_t waves = static_cast<int64_t>(gridDim.x) * (kBlock / kWave);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave; i < a.n; i += waves) {
        const T *x = static_cast<const T *>(a.x) + i * a.xs;
        const T *r = a.r ? static_cast<const T *>(a.r) + i * a.rs : nullptr;
        T *sum = a.sum ? static_cast<T *>(a.sum) + i * a.ss : nullptr;
        int8_t *q = a.q + i * a.qs;
        float top = 0.0f, squares = 0.0f;
        for (int d = lane; d < a.dim; d += kWave) {
            const float h = as_float(x[d]) + (r ? as_float(r[d]) : 0.0f);
            squares += h * h;
            top = max_nan(top, fabsf(a.w ? h * a.w[d] : h));
        }
        squares = group_sum<kWave>(squares);
        top = group_max_nan<kWave>(top);
        const float s = step_of(top), inv = inverse_step(s);
        for (int d = lane; d < round16(a.dim); d += kWave) {
            int b = 0;
            if (d < a.dim) {
                const float h = as_float(x[d]) + (r ? as_float(r[d]) : 0.0f);
                b = to_byte(a.w ? h * a.w[d] : h, inv);
                if (sum) sum[d] = from_float<T>(h);
            }
            q[d] = static_cast<int8_t>(b);
        }
        if (lane == 0) a.scale[i] = a.normalize ? s / sqrtf(squares / static_cast<float>(a.dim) + a.eps) : s;
    }
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
    const int64_t rows = kBlock / kWave;
    const int64_t blocks = (n + rows - 1) / rows;
    const unsigned grid = static_cast<unsigned>(blocks < (1 << 22) ? blocks : 1 << 22);
    if (dtype == TGL_OUT_F32) norm_kernel<float><<<grid, kBlock, 0, st>>>(a);
    else norm_kernel<bf16_t><<<grid, kBlock, 0, st>>>(a);
    return launch_status();
}

}  // extern "C"
