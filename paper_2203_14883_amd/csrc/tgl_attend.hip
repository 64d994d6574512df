// tgl_attend.hip -- attention of queries over a cache of keys and values in 8
// bits: out = sum_j exp(s_j) v_j / sum_j exp(s_j), s_j = scale <q, k_j>, over
// the positions that a query sees, in one pass with the running maximum and
// sum of the exponentials.
#include "tgl_cache.hpp"

namespace tgl {
namespace {

struct AttendArgs {
    CacheView c;
    SeqsView s;
    const int64_t *end;
    const void *q;
    void *out;
    float *lse;
    int64_t qt, qh, ot, oh;
    int64_t queries;
    int32_t q_heads;
    int32_t group;          // query heads of one head of the cache
    float scale;
};

// A wavefront per query and head: a token per lane for the scores, a column
// per lane for the output.
template <class T>
__global__ __launch_bounds__(kWave) void attend_kernel(const AttendArgs a) {
    __shared__ float qs[TGL_MAX_HEAD_DIM];
    __shared__ float ps[kWave];
    __shared__ int64_t at[kWave];
    const int lane = lane_id();
    const CacheView &c = a.c;
    const int64_t rows = a.s.seqs * a.queries * a.q_heads;
    for (int64_t u = blockIdx.x; u < rows; u += gridDim.x) {
        const int64_t row = u / a.q_heads, b = row / a.queries, t = row % a.queries;
        const int h = static_cast<int>(u % a.q_heads), head = h / a.group;
        const T *q = static_cast<const T *>(a.q) + row * a.qt + h * a.qh;
        __syncthreads();
        for (int d = lane; d < c.dim; d += kWave) qs[d] = as_float(q[d]) * a.scale;
        __syncthreads();
        const int64_t all = static_cast<int64_t>(a.s.pages_per_seq) << c.shift;
        int64_t begin = a.s.begin(b), end = a.end ? a.end[b] : all;
        end -= a.queries - 1 - t;
        begin = begin < 0 ? 0 : begin;
        end = end > all ? all : end;
        float m = -INFINITY;
        double l = 0.0;
        double o[TGL_MAX_HEAD_DIM / kWave] = {};
        for (int64_t j0 = begin; j0 < end; j0 += kWave) {
            const int64_t j = j0 + lane;
            const int64_t page = j < end ? a.s.page(b, j >> c.shift, c.pages) : -1;
            float s = -INFINITY, vs = 0.0f;
            if (page >= 0) {
                const int row_at = static_cast<int>(j & (c.tokens() - 1)) * c.width;
                const int8_t *k = c.rows(page, head, 0) + row_at;
                float dot = 0.0f;
                for (int d = 0; d < c.dim; d++) dot += qs[d] * static_cast<float>(k[d]);
                s = dot * *c.scale(page, head, 0);
                vs = *c.scale(page, head, 1);
                at[lane] = c.rows(page, head, 1) + row_at - c.data;
            }
            float top = s;
#pragma unroll
            for (int x = kWave / 2; x >= 1; x >>= 1) top = max_nan(top, __shfl_xor(top, x, kWave));
            const float next = max_nan(m, top);
            if (next == -INFINITY) continue;
            const float keep = m == -INFINITY ? 0.0f : expf(m - next);
            const float p = page >= 0 ? expf(s - next) : 0.0f;
            l = l * keep + group_sum<kWave>(p);
            m = next;
            ps[lane] = page >= 0 ? p * vs : 0.0f;
            if (page < 0) at[lane] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < TGL_MAX_HEAD_DIM / kWave; i++) {
                const int d = i * kWave + lane;
                if (d < c.dim) {
                    float sum = 0.0f;
                    for (int x = 0; x < kWave; x++) sum += ps[x] * static_cast<float>(c.data[at[x] + d]);
                    o[i] = o[i] * keep + sum;
                }
            }
            __syncthreads();
        }
        T *out = static_cast<T *>(a.out) + row * a.ot + h * a.oh;
#pragma unroll
        for (int i = 0; i < TGL_MAX_HEAD_DIM / kWave; i++) {
            const int d = i * kWave + lane;
            if (d < c.dim) out[d] = from_float<T>(m == -INFINITY ? 0.0f : static_cast<float>(o[i] / l));
        }
        if (a.lse && lane == 0) a.lse[row * a.q_heads + h] = m == -INFINITY ? -INFINITY : m + logf(static_cast<float>(l));
    }
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

size_t tgl_cache_attend_workspace(const tgl_cache *cache, const tgl_seqs *seqs, int32_t q_heads, int64_t queries) {
    (void)cache;
    (void)seqs;
    (void)q_heads;
    (void)queries;
    return 0;
}

tgl_status tgl_cache_attend(const tgl_cache *cache, const tgl_heads *q, int32_t q_heads, int64_t queries,
                            int32_t dtype, const tgl_seqs *seqs, const int64_t *end, float scale,
                            const tgl_heads *out, float *lse, void *workspace, size_t workspace_bytes,
                            void *stream) {
    if (!valid_cache(cache) || !valid_seqs(seqs) || seqs->offsets || !is_elem_type(dtype)) return TGL_EINVAL;
    if (q_heads < 1 || q_heads > TGL_MAX_HEADS || q_heads % cache->heads != 0 || queries < 1) return TGL_EINVAL;
    if (queries > (int64_t(1) << 31) || !aligned(end, 8) || !aligned(lse, 4) || !(scale == scale)) return TGL_EINVAL;
    const int64_t rows = seqs->num_seqs * queries;
    if (rows >= (int64_t(1) << 31)) return TGL_EINVAL;
    if (!valid_heads(q, rows, dtype) || !valid_heads(out, rows, dtype)) return TGL_EINVAL;
    if (workspace_bytes < tgl_cache_attend_workspace(cache, seqs, q_heads, queries)) return TGL_ENOSPACE;
    (void)workspace;
    if (rows == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const AttendArgs a{view_of(*cache), view_of(*seqs, rows), end, q->ptr, out->ptr, lse, q->token_stride, q->head_stride,
                       out->token_stride, out->head_stride, queries, q_heads, q_heads / cache->heads, scale};
    const int64_t work = rows * q_heads;
    const unsigned grid = static_cast<unsigned>(work < (1 << 22) ? work : 1 << 22);
    if (dtype == TGL_OUT_F32) attend_kernel<float><<<grid, kWave, 0, st>>>(a);
    else attend_kernel<bf16_t><<<grid, kWave, 0, st>>>(a);
    return launch_status();
}

}  // extern "C"
