// tgl_linear8.hip -- product of rows in 8 bits with a weight matrix in 8 bits:
//   out[i][j] = x_scale[i] * w_scale[j] * sum_k x[i][k] w[j][k] (+ bias[j])
// on the integer matrix instructions, whose int32 sums are exact.
#include "tgl_int8.hpp"

namespace tgl {
namespace {

struct LinearArgs {
    const int8_t *x;
    const int8_t *w;
    const float *xs;
    const float *ws;
    const float *bias;
    void *out;
    int64_t xstride, wstride, ostride;
    int64_t m;
    int32_t n, k;
};

// 16 consecutive bytes of a row from column c on, zeros from column k on.
// Rows are readable up to the next multiple of 16.
__device__ __forceinline__ i32x4 load_piece(const int8_t *row, int c, int k) {
    i32x4 v = {0, 0, 0, 0};
    if (c < k) v = *reinterpret_cast<const i32x4 *>(row + c);
    return v;
}

// The same with the bytes at and beyond column k cleared.
__device__ __forceinline__ i32x4 mask_piece(i32x4 v, int c, int k) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int left = k - (c + 4 * i);
        v[i] = left >= 4 ? v[i] : left <= 0 ? 0 : v[i] & static_cast<int>((1u << (8 * left)) - 1u);
    }
    return v;
}

// A wavefront per 16 x 16 outputs, operands straight from memory.
template <class T>
__global__ __launch_bounds__(kBlock) void linear_kernel(const LinearArgs a) {
    const int lane = lane_id();
    const int64_t tiles_n = (a.n + 15) / 16;
    const int64_t tile = static_cast<int64_t>(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave;
    if (tile >= (a.m + 15) / 16 * tiles_n) return;
    const int64_t m0 = tile / tiles_n * 16;
    const int n0 = static_cast<int>(tile % tiles_n) * 16;
    const int64_t mr = m0 + (lane & 15) < a.m ? m0 + (lane & 15) : a.m - 1;
    const int nr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const int8_t *x = a.x + mr * a.xstride;
    const int8_t *w = a.w + nr * a.wstride;
    i32x4 acc = {0, 0, 0, 0};
    for (int k = 0; k < a.k; k += 64) {
        const int c = k + 16 * (lane >> 4);
        const i32x4 av = mask_piece(load_piece(x, c, a.k), c, a.k);
        const i32x4 bv = load_piece(w, c, a.k);
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(av, bv, acc, 0, 0, 0);
    }
    const int col = n0 + (lane & 15);
    if (col >= a.n) return;
    const float ws = a.ws[col], b = a.bias ? a.bias[col] : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t row = m0 + 4 * (lane >> 4) + i;
        if (row < a.m) {
            const float y = static_cast<float>(acc[i]) * a.xs[row] * ws;
            static_cast<T *>(a.out)[row * a.ostride + col] = from_float<T>(a.bias ? y + b : y);
        }
    }
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

size_t tgl_linear_i8_workspace(int64_t m, int32_t n, int32_t k) {
    (void)m;
    (void)n;
    (void)k;
    return 0;
}

tgl_status tgl_linear_i8(const int8_t *x, int64_t x_stride, const float *x_scale, int64_t m, const int8_t *w,
                         int64_t w_stride, const float *w_scale, const float *bias, int32_t n, int32_t k,
                         void *out, int64_t out_stride, int32_t out_type, void *workspace,
                         size_t workspace_bytes, void *stream) {
    if (m < 0 || n < 1 || n > TGL_MAX_LINEAR_OUT || k < 1 || k > TGL_MAX_LINEAR_K || !is_elem_type(out_type))
        return TGL_EINVAL;
    if (!aligned(x, 16) || !aligned(w, 16) || x_stride % 16 != 0 || w_stride % 16 != 0 || x_stride < 0 || w_stride < 0)
        return TGL_EINVAL;
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(out, elem_size(out_type)))
        return TGL_EINVAL;
    if (m > 0 && (!x || !x_scale || !w || !w_scale || !out || out_stride < n)) return TGL_EINVAL;
    if (workspace_bytes < tgl_linear_i8_workspace(m, n, k)) return TGL_ENOSPACE;
    (void)workspace;
    if (m == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const LinearArgs a{x, w, x_scale, w_scale, bias, out, x_stride, w_stride, out_stride, m, n, k};
    const int64_t tiles = (m + 15) / 16 * ((n + 15) / 16);
    const int64_t blocks = (tiles + 3) / 4;
    if (blocks > 0x7fffffff) return TGL_EINVAL;
    const unsigned grid = static_cast<unsigned>(blocks);
    if (out_type == TGL_OUT_F32) linear_kernel<float><<<grid, kBlock, 0, st>>>(a);
    else linear_kernel<bf16_t><<<grid, kBlock, 0, st>>>(a);
    return launch_status();
}

}  // extern "C"
