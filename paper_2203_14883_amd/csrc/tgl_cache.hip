// tgl_cache.hip -- keys and values written to a cache in 8 bits, and read back.
//
// A page's head holds its keys (and its values) with one step, the largest
// magnitude among them over 127.  A page that is written in parts keeps one
// step: when new rows need a larger one, the rows that are there are rounded
// again.  One wavefront owns a page and head, so nothing is shared and no
// order matters.
#include "tgl_cache.hpp"

namespace tgl {
namespace {

struct IoArgs {
    CacheView c;
    SeqsView s;
    void *k;
    void *v;
    int64_t kt, kh, vt, vh;     // token and head strides
    int64_t items;              // write: page slots to look at
};

// Sequence b may touch the page slots (items) from base(b) on: cnt >= 1 tokens
// lie in at most (cnt + 2 P - 2) / P pages wherever they start, and the floors
// of sums below leave at least that many for each sequence.
__device__ __forceinline__ int64_t item_base(const SeqsView &s, int64_t b, int shift) {
    const int64_t P = int64_t(1) << shift;
    return (s.first_token(b) + b * (2 * P - 2)) >> shift;
}

// A wavefront per page slot and head, values in two passes over the new rows.
template <class T>
__global__ __launch_bounds__(kBlock) void write_kernel(const IoArgs a) {
    const int lane = lane_id();
    const CacheView &c = a.c;
    const int P = c.tokens(), D = c.dim, W = c.width;
    const int64_t waves = static_cast<int64_t>(gridDim.x) * (kBlock / kWave);
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave; u < a.items * c.heads; u += waves) {
        const int64_t item = u / c.heads;
        const int head = static_cast<int>(u % c.heads);
        int64_t lo = 0, hi = a.s.seqs;          // the last sequence whose items start at or before this one
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) / 2;
            if (item_base(a.s, mid, c.shift) <= item) lo = mid;
            else hi = mid;
        }
        const int64_t t0 = a.s.first_token(lo), t1 = a.s.first_token(lo + 1);
        const int64_t start = a.s.begin(lo);
        if (start < 0 || t1 <= t0) continue;
        const int64_t slot = (start >> c.shift) + (item - item_base(a.s, lo, c.shift));
        const int64_t p0 = slot << c.shift;                             // first position of the page
        const int64_t end = start + (t1 - t0);
        if (p0 >= end) continue;
        const int64_t page = a.s.page(lo, slot, c.pages);
        if (page < 0) continue;
        const int first = p0 < start ? static_cast<int>(start - p0) : 0;       // rows below are kept
        const int last = end - p0 < P ? static_cast<int>(end - p0) : P;
        const int64_t token = t0 + (p0 + first - start);
        for (int kind = 0; kind < 2; kind++) {
            const T *x = (kind ? static_cast<const T *>(a.v) + head * a.vh : static_cast<const T *>(a.k) + head * a.kh);
            const int64_t stride = kind ? a.vt : a.kt;
            int8_t *rows = c.rows(page, head, kind);
            float top = 0.0f;
            for (int r = first; r < last; r++)
                for (int d = lane; d < D; d += kWave) top = max_nan(top, fabsf(as_float(x[(token + r - first) * stride + d])));
            top = group_max_nan<kWave>(top);
            float s = step_of(top);
            const float old = *c.scale(page, head, kind);
            if (first > 0) s = max_nan(s, old);
            const float inv = inverse_step(s);
            for (int r = first; r < last; r++)
                for (int d = lane; d < W; d += kWave)
                    rows[r * W + d] = static_cast<int8_t>(d < D ? to_byte(as_float(x[(token + r - first) * stride + d]), inv) : 0);
            if (first > 0 && s != old) {
                const float f = old * inv;
                for (int d = lane; d < first * W; d += kWave) rows[d] = static_cast<int8_t>(to_byte(static_cast<float>(rows[d]), f));
            }
            if (lane == 0) *c.scale(page, head, kind) = s;
        }
    }
}

// A wavefront per token and head.
template <class T>
__global__ __launch_bounds__(kBlock) void read_kernel(const IoArgs a) {
    const int lane = lane_id();
    const CacheView &c = a.c;
    const int64_t waves = static_cast<int64_t>(gridDim.x) * (kBlock / kWave);
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave; u < a.s.tokens * c.heads; u += waves) {
        const int64_t token = u / c.heads;
        const int head = static_cast<int>(u % c.heads);
        int64_t lo = 0, hi = a.s.seqs;
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) / 2;
            if (a.s.first_token(mid) <= token) lo = mid;
            else hi = mid;
        }
        if (token < a.s.first_token(lo) || token >= a.s.first_token(lo + 1)) continue;
        const int64_t pos = a.s.begin(lo) + token - a.s.first_token(lo);
        const int64_t page = pos < 0 ? -1 : a.s.page(lo, pos >> c.shift, c.pages);
        const int row = static_cast<int>(pos & (c.tokens() - 1));
        for (int kind = 0; kind < 2; kind++) {
            T *x = (kind ? static_cast<T *>(a.v) + head * a.vh + token * a.vt : static_cast<T *>(a.k) + head * a.kh + token * a.kt);
            const int8_t *q = page < 0 ? nullptr : c.rows(page, head, kind) + row * c.width;
            const float s = page < 0 ? 0.0f : *c.scale(page, head, kind);
            for (int d = lane; d < c.dim; d += kWave) x[d] = from_float<T>(q ? static_cast<float>(q[d]) * s : 0.0f);
        }
    }
}

bool make_args(const tgl_cache *cache, const tgl_heads *k, const tgl_heads *v, int32_t dtype, int64_t num_tokens,
               const tgl_seqs *seqs, IoArgs *a) {
    if (!valid_cache(cache) || !is_elem_type(dtype) || num_tokens < 0 || !valid_seqs(seqs)) return false;
    if (!valid_heads(k, num_tokens, dtype) || !valid_heads(v, num_tokens, dtype)) return false;
    if (!seqs->offsets && (seqs->num_seqs ? num_tokens % seqs->num_seqs : num_tokens) != 0) return false;
    *a = IoArgs{view_of(*cache), view_of(*seqs, num_tokens), k->ptr, v->ptr, k->token_stride, k->head_stride,
                v->token_stride, v->head_stride, 0};
    return true;
}

unsigned grid_of(int64_t waves) {
    const int64_t blocks = (waves + kBlock / kWave - 1) / (kBlock / kWave);
    return static_cast<unsigned>(blocks < (1 << 22) ? blocks : 1 << 22);
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_cache_write(const tgl_cache *cache, const tgl_heads *k, const tgl_heads *v, int32_t dtype,
                           int64_t num_tokens, const tgl_seqs *seqs, void *stream) {
    IoArgs a;
    if (!make_args(cache, k, v, dtype, num_tokens, seqs, &a)) return TGL_EINVAL;
    if (num_tokens == 0 || seqs->num_seqs == 0 || cache->num_pages == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    a.items = ((num_tokens + seqs->num_seqs * (2 * int64_t(a.c.tokens()) - 2)) >> a.c.shift) + 1;
    const unsigned grid = grid_of(a.items * a.c.heads);
    if (dtype == TGL_OUT_F32) write_kernel<float><<<grid, kBlock, 0, st>>>(a);
    else write_kernel<bf16_t><<<grid, kBlock, 0, st>>>(a);
    return launch_status();
}

tgl_status tgl_cache_read(const tgl_cache *cache, const tgl_heads *k, const tgl_heads *v, int32_t out_type,
                          int64_t num_tokens, const tgl_seqs *seqs, void *stream) {
    IoArgs a;
    if (!make_args(cache, k, v, out_type, num_tokens, seqs, &a)) return TGL_EINVAL;
    if (num_tokens == 0 || seqs->num_seqs == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const unsigned grid = grid_of(num_tokens * a.c.heads);
    if (out_type == TGL_OUT_F32) read_kernel<float><<<grid, kBlock, 0, st>>>(a);
    else read_kernel<bf16_t><<<grid, kBlock, 0, st>>>(a);
    return launch_status();
}

}  // extern "C"
