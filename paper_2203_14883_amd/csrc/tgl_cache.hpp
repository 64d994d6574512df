// tgl_cache.hpp -- places of tokens in a cache of keys and values in 8 bits.
#pragma once

#include "tgl_int8.hpp"

namespace tgl {

struct CacheView {
    int8_t *data;
    float *scales;
    int64_t pages;
    int32_t shift;          // log2 of the tokens of a page
    int32_t heads;
    int32_t dim;
    int32_t width;          // dim rounded up to 16: bytes of a row

    __host__ __device__ int tokens() const { return 1 << shift; }
    // Bytes of the keys, or of the values, of one page and head.
    __host__ __device__ int64_t block_bytes() const { return static_cast<int64_t>(width) << shift; }
    __device__ int8_t *rows(int64_t page, int head, int kind) const {
        return data + ((page * heads + head) * 2 + kind) * block_bytes();
    }
    __device__ float *scale(int64_t page, int head, int kind) const { return scales + (page * heads + head) * 2 + kind; }
};

struct SeqsView {
    const int32_t *table;
    const int64_t *start;
    const int64_t *offsets;
    int64_t table_stride;
    int64_t per;            // tokens of every sequence, without offsets
    int64_t tokens;         // tokens of the call
    int32_t seqs;
    int32_t pages_per_seq;

    __device__ int64_t begin(int64_t b) const { return start ? start[b] : 0; }
    // The same between far below 0 and the table's end, so that sums with it stay whole numbers.
    __device__ int64_t bounded_begin(int64_t b, int shift) const {
        const int64_t v = begin(b), all = static_cast<int64_t>(pages_per_seq) << shift, low = -(int64_t(1) << 62);
        return v < low ? low : v > all ? all : v;
    }
    __device__ int64_t first_token(int64_t b) const {
        const int64_t t = offsets ? offsets[b] : b * per;
        return t < 0 ? 0 : t > tokens ? tokens : t;
    }
    // The page of a sequence's i-th page slot, or -1.
    __device__ int64_t page(int64_t b, int64_t i, int64_t pages) const {
        if (i < 0 || i >= pages_per_seq) return -1;
        const int64_t p = table[b * table_stride + i];
        return p >= 0 && p < pages ? p : -1;
    }
};

inline CacheView view_of(const tgl_cache &c) {
    int shift = 0;
    while ((1 << shift) < c.page_tokens) shift++;
    return CacheView{c.data, c.scales, c.num_pages, shift, c.heads, c.dim, round16(c.dim)};
}

inline SeqsView view_of(const tgl_seqs &s, int64_t tokens) {
    return SeqsView{s.table, s.start, s.offsets, s.table_stride, s.num_seqs ? tokens / s.num_seqs : 0, tokens,
                    static_cast<int32_t>(s.num_seqs), s.pages_per_seq};
}

}  // namespace tgl
