// tgl_cache.hip -- keys and values written to a cache in 8 bits, and read back.
//
// A page's head holds its keys (and its values) with one step, the largest
// magnitude among them over 127.  A page that is written in parts keeps one
// step: when new rows need a larger one, the rows that are there are rounded
// again.  One group of lanes owns the keys, or the values, of a page and head,
// so nothing is shared and no order matters.  Both directions only move bytes:
// new rows are read once, into registers, and written as soon as their
// largest magnitude is known.
#include "tgl_cache.hpp"

namespace tgl {
namespace {

constexpr int kRun = 8;             // elements of a lane's access
constexpr int64_t kFill = 16384;    // wavefronts that fill the card four times over

struct IoArgs {
    CacheView c;
    SeqsView s;
    void *k;
    void *v;
    int64_t kt, kh, vt, vh;         // token and head strides
    int64_t units;                  // write: page slots to look at, times parts
    int32_t parts, pairs;           // write: 2 heads = parts * pairs
    Div runs;                       // write: whole runs of a row (1 for none); read: runs of a row's elements
    int32_t whole;                  // write: whole runs of a row
    Div row_runs;                   // read: runs of a token, all heads
    int32_t block_tokens;           // read: tokens of a workgroup
};

// Sequence b may touch the page slots (items) from base(b) on: cnt >= 1 tokens
// lie in at most (cnt + 2 P - 2) / P pages wherever they start, and the floors
// of sums below leave at least that many for each sequence.
__device__ __forceinline__ int64_t item_base(const SeqsView &s, int64_t b, int shift) {
    const int64_t P = int64_t(1) << shift;
    return (s.first_token(b) + b * (2 * P - 2)) >> shift;
}

// The last sequence whose items start at or before this one; the G lanes of a
// group look at G places at a time.
template <int G>
__device__ __forceinline__ int64_t find_sequence(const SeqsView &s, int64_t item, int shift, int i) {
    int64_t lo = 0, hi = s.seqs;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + G - 1) / G;
        const int64_t at = lo + i * step;
        const bool before = at < hi && item_base(s, at, shift) <= item;
        const uint64_t found = group_ballot<G>(before);
        const int n = __popcll(found);
        lo += (n > 0 ? n - 1 : 0) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

// L lanes own a unit: a.pairs of the 2 heads keys and values of a page slot, one
// after another, so that a place is looked up once for all of them.  Up to
// kHold runs of 8 elements a lane stay in registers between the two looks at
// them; what does not fit (pages that fill up beyond the call's average) is
// read again.  Bound by memory once enough of it is in flight: 307,000 tokens of
// 8 heads of 128 bfloat16 in pages of 32 (1.26 GB read, 0.63 written) 432 us,
// 4.4 TB/s; 600 us without the next ones on their way, 1520 us in two passes
// over the rows.  One token for each of 4000 histories 13.8 us: the chain of
// looking places up.
template <class T, int L>
__global__ __launch_bounds__((L > kBlock ? L : kBlock), 4) void write_kernel(const IoArgs a) {
    constexpr int kHold = sizeof(T) == 2 ? 4 : 2;       // 16 registers
    constexpr int kGroup = L > kWave ? kWave : L;
    constexpr int kUnits = L > kBlock ? 1 : kBlock / L;                 // of a workgroup
    __shared__ float tops[L / kWave + 1];
    const CacheView &c = a.c;
    const int P = c.tokens(), D = c.dim, W = c.width;
    const int i = threadIdx.x % L;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kUnits;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * kUnits + threadIdx.x / L; u - threadIdx.x / L < a.units; u += stride) {
        // every lane stays for the exchanges below: without work, it has no rows
        const int64_t unit = u < a.units ? u : a.units - 1;
        const int64_t item = unit / a.parts;
        const int pair0 = static_cast<int>(unit - item * a.parts) * a.pairs;
        const int64_t b = find_sequence<kGroup>(a.s, item, c.shift, threadIdx.x % kGroup);
        const int64_t t0 = a.s.first_token(b), t1 = a.s.first_token(b + 1);
        const int64_t start = a.s.bounded_begin(b, c.shift);
        const int64_t slot = (start >> c.shift) + (item - item_base(a.s, b, c.shift));
        const int64_t p0 = slot << c.shift;                             // first position of the page
        const int64_t end = start + (t1 - t0);
        int64_t page = -1;
        if (u < a.units && start >= 0 && t1 > t0 && p0 < end) page = a.s.page(b, slot, c.pages);
        const int first = page >= 0 && p0 < start ? static_cast<int>(start - p0) : 0;      // rows below are kept
        const int rows = page < 0 ? 0 : static_cast<int>((end - p0 < P ? end - p0 : P) - first);
        const int64_t token = t0 + (p0 + first - start);
        const int runs = rows * a.runs.d * (a.whole > 0 ? 1 : 0);      // whole runs; what is left of a row comes by itself
        const int tail = a.whole * kRun;

        auto rows_of = [&](int pair) {
            return pair & 1 ? static_cast<const T *>(a.v) + (pair >> 1) * a.vh + token * a.vt
                            : static_cast<const T *>(a.k) + (pair >> 1) * a.kh + token * a.kt;
        };
        auto run_at = [&](const T *x, int pitch, int n) {
            const int r = a.runs(n);
            return reinterpret_cast<const Run<T, kRun> *>(x + (static_cast<int64_t>(r) * pitch + (n - r * a.runs.d) * kRun));
        };
        auto fetch = [&](int pair, Run<T, kRun> (&held)[kHold], float &old) {
            const T *x = rows_of(pair);
            const int pitch = static_cast<int>(pair & 1 ? a.vt : a.kt);
#pragma unroll
            for (int h = 0; h < kHold; h++)
                if (i + h * L < runs) held[h] = *run_at(x, pitch, i + h * L);
            old = first > 0 ? *c.scale(page, pair >> 1, pair & 1) : 0.0f;
        };
        Run<T, kRun> held[kHold], next[kHold];
        float old, next_old = 0.0f;
        fetch(pair0, held, old);
        for (int pair = pair0; pair < pair0 + a.pairs; pair++) {
            // the next keys or values are on their way while these are rounded
            if (pair + 1 < pair0 + a.pairs) fetch(pair + 1, next, next_old);
            const T *x = rows_of(pair);
            const int pitch = static_cast<int>(pair & 1 ? a.vt : a.kt);
            uint32_t bits = 0;          // of the largest magnitude: NaN above infinity above numbers
            auto look = [&](float v) {
                const uint32_t w = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
                bits = w > bits ? w : bits;
            };
#pragma unroll
            for (int h = 0; h < kHold; h++)
                if (i + h * L < runs)
                    for (int k = 0; k < kRun; k++) look(as_float(held[h].t[k]));
            for (int n = i + kHold * L; n < runs; n += L) {
                const Run<T, kRun> w = *run_at(x, pitch, n);
#pragma unroll
                for (int k = 0; k < kRun; k++) look(as_float(w.t[k]));
            }
            if (tail < D)
                for (int r = i; r < rows; r += L)
                    for (int d = tail; d < D; d++) look(as_float(x[static_cast<int64_t>(r) * pitch + d]));
#pragma unroll
            for (int d = kGroup / 2; d >= 1; d >>= 1) {
                const uint32_t v = __shfl_xor(bits, d, kWave);
                bits = v > bits ? v : bits;
            }
            if constexpr (L > kWave) {
                __syncthreads();        // the last ones' readers are done
                if (lane_id() == 0) tops[threadIdx.x / kWave] = __builtin_bit_cast(float, bits);
                __syncthreads();
#pragma unroll
                for (int w = 0; w < L / kWave; w++) {
                    const uint32_t v = __builtin_bit_cast(uint32_t, tops[threadIdx.x / L * (L / kWave) + w]);
                    bits = v > bits ? v : bits;
                }
            }
            float s = step_of(__builtin_bit_cast(float, bits));
            if (first > 0) s = max_nan(s, old);
            const float inv = inverse_step(s);
            int8_t *out = c.rows(page < 0 ? 0 : page, pair >> 1, pair & 1);
            auto put = [&](int8_t *at, const Run<T, kRun> &w) {
                i32x2 v = {0, 0};
                if (inv != 0.0f)
                    v = i32x2{to_bytes4(as_float(w.t[0]), as_float(w.t[1]), as_float(w.t[2]), as_float(w.t[3]), inv),
                              to_bytes4(as_float(w.t[4]), as_float(w.t[5]), as_float(w.t[6]), as_float(w.t[7]), inv)};
                *reinterpret_cast<i32x2 *>(at) = v;
            };
            auto place = [&](int n) {
                const int r = a.runs(n);
                return out + ((first + r) * W + (n - r * a.runs.d) * kRun);
            };
#pragma unroll
            for (int h = 0; h < kHold; h++)
                if (i + h * L < runs) put(place(i + h * L), held[h]);
            for (int n = i + kHold * L; n < runs; n += L) put(place(n), *run_at(x, pitch, n));
            if (tail < W) {
                for (int r = i; r < rows; r += L) {
                    for (int d = tail; d < W; d += kRun) {
                        Run<T, kRun> w;
#pragma unroll
                        for (int k = 0; k < kRun; k++) w.t[k] = d + k < D ? x[static_cast<int64_t>(r) * pitch + d + k] : from_float<T>(0.0f);
                        put(out + ((first + r) * W + d), w);
                    }
                }
            }
            if (rows > 0 && first > 0 && s != old) {
                const float f = old * inv;
                for (int n = i; n < first * (W / kRun); n += L) {
                    i32x2 *at = reinterpret_cast<i32x2 *>(out + n * kRun);
                    i32x2 v = *at;
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        const int word = v[k];
                        const float q[4] = {static_cast<float>(static_cast<int8_t>(word)), static_cast<float>(static_cast<int8_t>(word >> 8)),
                                            static_cast<float>(static_cast<int8_t>(word >> 16)), static_cast<float>(word >> 24)};
                        v[k] = f > 0.0f ? to_bytes4(q[0], q[1], q[2], q[3], f) : 0;
                    }
                    *at = v;
                }
            }
            if (rows > 0 && i == 0) *c.scale(page, pair >> 1, pair & 1) = s;
#pragma unroll
            for (int h = 0; h < kHold; h++) held[h] = next[h];
            old = next_old;
        }
    }
}

// The last sequence whose tokens start at or before this one (a wavefront).
__device__ __forceinline__ int64_t last_at_most(const SeqsView &s, int64_t token) {
    int64_t lo = 0, hi = s.seqs;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave;
        const int64_t at = lo + lane_id() * step;
        const int n = __popcll(__ballot(at < hi && s.first_token(at) <= token));
        lo += (n > 0 ? n - 1 : 0) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

// A workgroup takes block_tokens tokens in turn: a thread each looks one up,
// then all stream its heads, 16 bytes of keys and of values a lane, past the
// caches.  Bound by memory: the tokens above read back (0.63 GB read, 1.26
// written) in 374 us, 5.1 TB/s; 120,000 slots of 2 heads of 50 float32 from 2M
// one-token pages in 39 us, 42 MB read and 123 written (96 of them numbers: rows
// of 200 bytes leave lines that are written in parts), 4.2 TB/s (50 us
// with stores of 32 bytes a lane through the caches).
template <class T>
__global__ __launch_bounds__(kBlock) void read_kernel(const IoArgs a) {
    constexpr int kRead = 16 / sizeof(T);       // elements of a lane's stores
    __shared__ int at_page[kBlock];
    __shared__ int at_row[kBlock];
    __shared__ int64_t ends[2];
    const CacheView &c = a.c;
    const int B = a.block_tokens;
    const int64_t blocks = (a.s.tokens + B - 1) / B;
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const int64_t base = block * B;
        const int count = a.s.tokens - base < B ? static_cast<int>(a.s.tokens - base) : B;
        __syncthreads();
        // the sequences of the first and of the last token, 64 places at a time
        if (a.s.offsets) {
            if (threadIdx.x < 2 * kWave) {
                const int last = threadIdx.x / kWave;
                const int64_t b = last_at_most(a.s, last ? base + count - 1 : base);
                if (lane_id() == 0) ends[last] = b;
            }
            __syncthreads();
        }
        if (static_cast<int>(threadIdx.x) < count) {
            const int64_t token = base + threadIdx.x;
            int64_t b = 0;
            if (a.s.offsets) {
                int64_t lo = ends[0], hi = ends[1] + 1;
                while (hi - lo > 1) {
                    const int64_t mid = (lo + hi) / 2;
                    if (a.s.first_token(mid) <= token) lo = mid;
                    else hi = mid;
                }
                b = lo;
            } else {
                b = token / a.s.per;
            }
            int page = -2;                                              // no sequence's
            int row = 0;
            if (token >= a.s.first_token(b) && token < a.s.first_token(b + 1)) {
                const int64_t pos = a.s.bounded_begin(b, c.shift) + token - a.s.first_token(b);
                page = pos < 0 ? -1 : static_cast<int>(a.s.page(b, pos >> c.shift, c.pages));
                row = static_cast<int>(pos) & (c.tokens() - 1);
            }
            at_page[threadIdx.x] = page;
            at_row[threadIdx.x] = row;
        }
        __syncthreads();
        const int total = count * a.row_runs.d;
#pragma unroll 4
        for (int n = threadIdx.x; n < total; n += kBlock) {
            const int t = a.row_runs(n);
            const int rest = n - t * a.row_runs.d;
            const int head = a.runs(rest);
            const int d = (rest - head * a.runs.d) * kRead;
            const int page = at_page[t];
            if (page == -2) continue;
            const int own = page < 0 ? 0 : page;
            Columns<kRead> kq = {}, vq = {};
            float2 s = {0.0f, 0.0f};
            if (c.pages > 0) {
                const int8_t *q = c.rows(own, head, 0) + at_row[t] * c.width + d;
                kq.load(q);
                vq.load(q + c.block_bytes());
                s = *reinterpret_cast<const float2 *>(c.scale(own, head, 0));
            }
            float k[kRead], v[kRead];
#pragma unroll
            for (int e = 0; e < kRead; e++) {
                k[e] = page < 0 ? 0.0f : static_cast<float>(static_cast<int8_t>(kq.w[e / 4] >> (8 * (e % 4)))) * s.x;
                v[e] = page < 0 ? 0.0f : static_cast<float>(static_cast<int8_t>(vq.w[e / 4] >> (8 * (e % 4)))) * s.y;
            }
            store_columns<T, kRead, true>(static_cast<T *>(a.k) + (base + t) * a.kt + head * a.kh, d, c.dim, k);
            store_columns<T, kRead, true>(static_cast<T *>(a.v) + (base + t) * a.vt + head * a.vh, d, c.dim, v);
        }
    }
}

bool make_args(const tgl_cache *cache, const tgl_heads *k, const tgl_heads *v, int32_t dtype, int64_t num_tokens,
               const tgl_seqs *seqs, IoArgs *a) {
    if (!valid_cache(cache) || !is_elem_type(dtype) || num_tokens < 0 || !valid_seqs(seqs)) return false;
    if (!valid_heads(k, num_tokens, dtype) || !valid_heads(v, num_tokens, dtype)) return false;
    if (!seqs->offsets && (seqs->num_seqs ? num_tokens % seqs->num_seqs : num_tokens) != 0) return false;
    *a = IoArgs{};
    a->c = view_of(*cache);
    a->s = view_of(*seqs, num_tokens);
    a->k = k->ptr;
    a->v = v->ptr;
    a->kt = k->token_stride;
    a->kh = k->head_stride;
    a->vt = v->token_stride;
    a->vh = v->head_stride;
    return true;
}

unsigned grid_of(int64_t blocks) { return static_cast<unsigned>(blocks < (1 << 22) ? blocks : 1 << 22); }

template <class T, int L>
void launch_write(IoArgs a, int64_t items, hipStream_t st) {
    // as many keys and values a unit as leave kFill wavefronts, up to 8
    constexpr int kBlockOf = L > kBlock ? L : kBlock;
    a.parts = 2 * a.c.heads;
    a.pairs = 1;
    while (a.pairs < 8 && a.parts % 2 == 0 && items * (a.parts / 2) * L >= kFill * kWave) {
        a.parts /= 2;
        a.pairs *= 2;
    }
    a.units = items * a.parts;
    write_kernel<T, L><<<grid_of((a.units * L + kBlockOf - 1) / kBlockOf), kBlockOf, 0, st>>>(a);
}

// Lanes of a unit by the runs of the rows that it gets on average.
template <class T>
void launch_write(const IoArgs &a, int64_t items, int64_t rows, hipStream_t st) {
    const int64_t runs = rows * (a.c.width / kRun);
    if (runs <= 32) launch_write<T, 16>(a, items, st);
    else if (runs <= 256) launch_write<T, 64>(a, items, st);
    else if (runs <= 1024) launch_write<T, 256>(a, items, st);
    else launch_write<T, 512>(a, items, st);
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_cache_write(const tgl_cache *cache, const tgl_heads *k, const tgl_heads *v, int32_t dtype,
                           int64_t num_tokens, const tgl_seqs *seqs, void *stream) {
    IoArgs a;
    if (!make_args(cache, k, v, dtype, num_tokens, seqs, &a)) return TGL_EINVAL;
    // a row's place in its page is found with 32 bits
    if (k->token_stride != static_cast<int32_t>(k->token_stride) || v->token_stride != static_cast<int32_t>(v->token_stride))
        return TGL_EINVAL;
    if (num_tokens == 0 || seqs->num_seqs == 0 || cache->num_pages == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const int64_t P = a.c.tokens();
    const int64_t items = ((num_tokens + seqs->num_seqs * (2 * P - 2)) >> a.c.shift) + 1;
    a.whole = a.c.dim / kRun;
    a.runs = Div(a.whole > 0 ? a.whole : 1);
    const int64_t each = (num_tokens + seqs->num_seqs - 1) / seqs->num_seqs;
    const int64_t rows = each < P ? each : P;
    if (dtype == TGL_OUT_F32) launch_write<float>(a, items, rows, st);
    else launch_write<bf16_t>(a, items, rows, st);
    return launch_status();
}

tgl_status tgl_cache_read(const tgl_cache *cache, const tgl_heads *k, const tgl_heads *v, int32_t out_type,
                          int64_t num_tokens, const tgl_seqs *seqs, void *stream) {
    IoArgs a;
    if (!make_args(cache, k, v, out_type, num_tokens, seqs, &a)) return TGL_EINVAL;
    if (num_tokens == 0 || seqs->num_seqs == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const int run = 16 / static_cast<int>(elem_size(out_type));
    a.runs = Div((a.c.dim + run - 1) / run);
    a.row_runs = Div(a.runs.d * a.c.heads);
    // tokens of a workgroup: about 16 runs a thread, fewer where that would leave compute units idle
    int64_t tokens = 16 * kBlock / a.row_runs.d;
    const int64_t most = num_tokens / 2048;
    tokens = tokens > most ? most : tokens;
    a.block_tokens = static_cast<int32_t>(tokens < 1 ? 1 : tokens > kBlock ? kBlock : tokens);
    const unsigned grid = grid_of((num_tokens + a.block_tokens - 1) / a.block_tokens);
    if (out_type == TGL_OUT_F32) read_kernel<float><<<grid, kBlock, 0, st>>>(a);
    else read_kernel<bf16_t><<<grid, kBlock, 0, st>>>(a);
    return launch_status();
}

}  // extern "C"
