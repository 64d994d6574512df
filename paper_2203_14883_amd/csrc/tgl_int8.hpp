// tgl_int8.hpp -- what the 8-bit operators share: element types, the rounding
// of a set of numbers to bytes and a step, wide accesses, argument checks.
#pragma once

#include "tgl_internal.hpp"

namespace tgl {

using i32x4 = int __attribute__((ext_vector_type(4)));
using i32x2 = int __attribute__((ext_vector_type(2)));
using f32x4 = float __attribute__((ext_vector_type(4)));

struct bf16_t {
    uint16_t bits;
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16_t v) { return __builtin_bit_cast(float, static_cast<uint32_t>(v.bits) << 16); }

template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t from_float<bf16_t>(float v) {
    return bf16_t{__builtin_bit_cast(uint16_t, static_cast<__bf16>(v))};
}

// ---- a set of numbers in 8 bits ----

constexpr float kTiny = 0x1p-100f;      // sets whose largest magnitude is below have step 0

// The larger of two magnitudes, NaN if either is (fmaxf drops a NaN).
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

// The step of a set whose largest magnitude is a (NaN if there was one).
__device__ __forceinline__ float step_of(float a) {
    if (!(a <= 3.4028235e38f)) return __builtin_nanf("");
    return a < kTiny ? 0.0f : a * (1.0f / 127.0f);
}

// 1 / s, or 0 where every byte is to be 0 (a step of 0 or NaN).
__device__ __forceinline__ float inverse_step(float s) { return s > 0.0f ? 1.0f / s : 0.0f; }

// ---- loops over constants ----

// f(0), f(1), ... f(N - 1) with constant arguments.
template <int K>
struct Const {
    static constexpr int value = K;
};
template <int N, int K = 0, class F>
__device__ __forceinline__ void unrolled(const F &f) {
    if constexpr (K < N) {
        f(Const<K>());
        unrolled<N, K + 1>(f);
    }
}

// ---- wide accesses ----

// N consecutive elements that need not lie at a multiple of their size: one
// wide access wherever they start.
template <class T, int N>
struct __attribute__((packed, aligned(alignof(T)))) Run {
    T t[N];
};

// N elements of a row from column d on, zeros from column dim on.
template <class T, int N>
__device__ __forceinline__ void load_columns(const T *q, int d, int dim, float (&x)[N]) {
    if (d + N <= dim) {
        const Run<T, N> w = *reinterpret_cast<const Run<T, N> *>(q + d);
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = as_float(w.t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float v = as_float(q[d + i < dim ? d + i : dim - 1]);
            x[i] = d + i < dim ? v : 0.0f;
        }
    }
}

// N consecutive elements from column d on, as far as there are columns; kStream:
// N are 16 bytes that nothing nearby reads again.
template <class T, int N, bool kStream = false>
__device__ __forceinline__ void store_columns(T *out, int d, int dim, const float (&x)[N]) {
    if (d + N <= dim) {
        Run<T, N> w;
#pragma unroll
        for (int i = 0; i < N; i++) w.t[i] = from_float<T>(x[i]);
        if constexpr (kStream) {
            using word_t = i32x4 __attribute__((aligned(alignof(T))));
            __builtin_nontemporal_store(__builtin_bit_cast(i32x4, w), reinterpret_cast<word_t *>(out + d));
        } else {
            *reinterpret_cast<Run<T, N> *>(out + d) = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
            if (d + i < dim) out[d + i] = from_float<T>(x[i]);
    }
}

// JV bytes of a row (a multiple of JV from its start), as whole dwords.
template <int JV>
struct Columns {
    static constexpr int kWords = JV >= 4 ? JV / 4 : 1;
    int w[kWords];
    __device__ __forceinline__ void load(const int8_t *p) {
        if constexpr (JV == 2) w[0] = *reinterpret_cast<const uint16_t *>(p);
        if constexpr (JV == 4) w[0] = *reinterpret_cast<const int *>(p);
        if constexpr (JV == 8) {
            const i32x2 v = *reinterpret_cast<const i32x2 *>(p);
            w[0] = v[0];
            w[1] = v[1];
        }
        if constexpr (JV == 16) {
            const i32x4 v = *reinterpret_cast<const i32x4 *>(p);
            for (int i = 0; i < 4; i++) w[i] = v[i];
        }
    }
};

// Four numbers in units of a step, as the bytes of a word.  Adding 1.5 * 2^23
// rounds a number to whole ones (ties to even, as rint does) and leaves it in
// the low bits.  inv must not be 0: the caller writes zeros there.
__device__ __forceinline__ int to_bytes4(float a, float b, float c, float d, float inv) {
    constexpr float kRound = 12582912.0f;
    const int ia = __builtin_bit_cast(int, a * inv + kRound), ib = __builtin_bit_cast(int, b * inv + kRound);
    const int ic = __builtin_bit_cast(int, c * inv + kRound), id = __builtin_bit_cast(int, d * inv + kRound);
    const int ab = __builtin_amdgcn_perm(ib, ia, 0x0c0c0400u), cd = __builtin_amdgcn_perm(id, ic, 0x0c0c0400u);
    return ab | (cd << 16);
}

// Division of whole numbers below 2^31 by a fixed one: with 2^l >= d and
// mul = ceil(2^(31+l) / d) the quotient is n mul >> (31 + l), exactly.
struct Div {
    uint32_t mul = 0, shift = 0, d = 1;
    Div() = default;
    explicit Div(uint32_t by) : d(by) {
        int l = 0;
        while ((uint64_t(1) << l) < by) l++;
        shift = 31 + l;
        mul = static_cast<uint32_t>(((uint64_t(1) << shift) + by - 1) / by);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
        return static_cast<uint32_t>((static_cast<uint64_t>(n) * mul) >> shift);
    }
};

// ---- host side ----

inline bool is_elem_type(int32_t t) { return t == TGL_OUT_F32 || t == TGL_OUT_BF16; }
inline size_t elem_size(int32_t t) { return t == TGL_OUT_F32 ? 4 : 2; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
__host__ __device__ inline int32_t round16(int32_t d) { return (d + 15) & ~15; }

inline bool valid_cache(const tgl_cache *c) {
    return c && c->num_pages >= 0 && c->num_pages < (int64_t(1) << 31) && c->page_tokens >= 1 &&
           c->page_tokens <= TGL_MAX_PAGE && (c->page_tokens & (c->page_tokens - 1)) == 0 && c->heads >= 1 &&
           c->heads <= TGL_MAX_HEADS && c->dim >= 1 && c->dim <= TGL_MAX_HEAD_DIM && c->reserved == 0 &&
           (c->num_pages == 0 || (c->data && c->scales)) && aligned(c->data, 16) && aligned(c->scales, 8);
}

inline bool valid_seqs(const tgl_seqs *s) {
    return s && s->num_seqs >= 0 && s->num_seqs < (int64_t(1) << 31) && s->pages_per_seq >= 0 && s->reserved == 0 &&
           s->table_stride >= 0 && (s->num_seqs == 0 || s->pages_per_seq == 0 || s->table) && aligned(s->table, 4) &&
           aligned(s->start, 8) && aligned(s->offsets, 8);
}

// Rows of heads whose elements have that type; strides may be 0 or negative for inputs.
inline bool valid_heads(const tgl_heads *h, int64_t rows, int32_t dtype) {
    return h && (rows == 0 || h->ptr) && aligned(h->ptr, elem_size(dtype));
}

}  // namespace tgl
