// tgl_attend.hip -- attention of queries over a cache of keys and values in 8
// bits: out = sum_j exp(s_j) v_j / sum_j exp(s_j), s_j = scale <q, k_j>, over
// the positions that a query sees, in one pass with the running maximum and
// sum of the exponentials.
//
// The queries that read one head of the cache (its group of query heads, for
// every query of the sequence) are rows; 16 of them make a row tile, and a
// wavefront takes 32 tokens at a time against it:
//
//   scores  S^T = K Q^T on the int8 matrix instructions.  The keys go in as
//           they lie in the cache; a query row goes in as two signed bytes of
//           a 16-bit whole number (bfloat16 queries) or three of a 24-bit one
//           (float32), in units of its largest element / (127 * 256^(n-1)).
//           The sums are exact; what is lost is that rounding, 2^-16 or 2^-24
//           of the row's largest element.
//   output  O^T = V^T P^T on the f16 ones.  S^T leaves every lane four tokens
//           of a row per 16 x 16 tile, which is what P^T takes with the tokens
//           in a fixed other order, so the probabilities never leave their
//           lane.  V^T wants, per lane, one column of eight tokens: a lane
//           loads the same few columns of its eight tokens and picks a
//           column's bytes with v_perm.  A byte b ^ 0x80 = v + 128 read as the bits
//           of an f16 is (v + 128) 2^-24, and one packed fused multiply-add
//           makes it v 2^-9, exactly.
//   P       carries the step of its token's page over the largest step seen so
//           far (a running one, like the maximum), so that pages of any steps
//           add up.  P is f16: one for bfloat16 outputs (2^-11 of each), two,
//           the second the rounding error of the first, for float32.
#include "tgl_cache.hpp"

namespace tgl {
namespace {

using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

constexpr int kRows = 16;           // rows of a tile
constexpr int kTile = 32;           // tokens of a wavefront's step
constexpr float kLog2E = 1.44269504088896340736f;

struct AttendArgs {
    CacheView c;
    SeqsView s;
    const int64_t *end;
    const void *q;
    void *out;
    float *lse;
    float *part_o;          // [rows of all heads][chunks][dim], or null
    float *part_ml;         // [rows of all heads][chunks][2]
    int64_t qt, qh, ot, oh;
    int64_t queries;
    int64_t row_tiles;      // of one sequence and head
    int64_t chunk;          // tokens of a workgroup
    int64_t work;           // workgroups
    int32_t chunks;
    int32_t group;          // query heads of one head of the cache
    float scale;
};

// What a lane knows of its row: the query, the head, whether it exists.
struct Row {
    int64_t q;              // row of q and out
    int32_t head;           // query head
    bool there;
};

__device__ __forceinline__ Row row_of(const AttendArgs &a, int64_t b, int head, int64_t r) {
    const int64_t t = r / a.group;
    return Row{b * a.queries + t, static_cast<int32_t>(head * a.group + (r - t * a.group)), r < a.queries * a.group};
}

template <class T>
constexpr int kParts = 2;           // bytes of a query element
template <>
constexpr int kParts<float> = 3;

// Largest log2 of a weight relative to the running maximum before that is
// raised, and the offset of all of them, so that f16 holds at most 2^14 (2^15
// with a step that is up to twice the running one).
template <class T>
constexpr float kSlack = 8.0f;
template <>
constexpr float kSlack<float> = 1.0f;
template <class T>
constexpr float kOffset = 14.0f - kSlack<T>;

// The row's query as signed bytes, kk-th piece of 64 columns, part p; returns
// the size of one unit.
template <class T, int KK>
__device__ __forceinline__ float load_query(const AttendArgs &a, const Row &row, int lane, i32x4 (&parts)[kParts<T>][KK]) {
    constexpr int N = kParts<T>;
    const T *q = static_cast<const T *>(a.q) + row.q * a.qt + row.head * a.qh;
    float x[KK][16];
    float top = 0.0f;
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int d = 64 * kk + 16 * (lane >> 4) + i;
            x[kk][i] = row.there && d < a.c.dim ? as_float(q[d]) : 0.0f;
            top = max_nan(top, fabsf(x[kk][i]));
        }
    }
    top = max_nan(top, __shfl_xor(top, 16, kWave));
    top = max_nan(top, __shfl_xor(top, 32, kWave));
    constexpr float kUnits = N == 2 ? 127.0f * 256.0f : 127.0f * 65536.0f;
    // not finite: a NaN unit makes the row NaN; tiny: zeros
    const float unit = !(top <= 3.4028235e38f) ? __builtin_nanf("") : top < kTiny ? 0.0f : top / kUnits;
    const float inv = inverse_step(unit);
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
#pragma unroll
        for (int w = 0; w < 4; w++) {
            int word[N] = {};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                int v = to_byte(x[kk][4 * w + i], inv);
#pragma unroll
                for (int p = N - 1; p >= 0; p--) {
                    const int low = static_cast<int8_t>(v);
                    word[p] |= (low & 255) << (8 * i);
                    v = (v - low) >> 8;
                }
            }
#pragma unroll
            for (int p = 0; p < N; p++) parts[p][kk][w] = word[p];
        }
    }
    return unit;
}

// JV columns of values of a token, as whole dwords.
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

// Column jj of a word of two tokens, as f16: (v + 128) 2^-24 -> v 2^-9.
__device__ __forceinline__ int column_pair(int a, int b, int jj) {
    const unsigned sel = 0x0c000c00u | (static_cast<unsigned>(4 + jj) << 16) | static_cast<unsigned>(jj);
    const f16x2 u = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(b, a, sel));
    const f16x2 up = {static_cast<_Float16>(32768.0f), static_cast<_Float16>(32768.0f)};
    const f16x2 off = {static_cast<_Float16>(-0.25f), static_cast<_Float16>(-0.25f)};
    return __builtin_bit_cast(int, __builtin_elementwise_fma(u, up, off));
}

__device__ __forceinline__ int pack_f16(float a, float b) {
    return __builtin_bit_cast(int, f16x2{static_cast<_Float16>(a), static_cast<_Float16>(b)});
}

// JV: columns of a lane, so heads of up to 16 JV.  kWhole: pages of at least
// 16 tokens, one page to each half of a step.  NW: wavefronts that share a
// workgroup's tokens.
template <class T, int JV, bool kWhole, int NW>
__global__ __launch_bounds__(NW * kWave) void attend_kernel(const AttendArgs a) {
    constexpr int N = kParts<T>;
    constexpr int KK = JV >= 4 ? JV / 4 : 1;
    const CacheView &c = a.c;
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int g = lane >> 4, i16 = lane & 15;
    // a contiguous stretch of the work for each of the 8 dies, whose L2 then
    // serves the row tiles of one head
    const int64_t per = (a.work + 7) / 8;
    const int64_t id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || id >= a.work) return;
    const int64_t tile = id % a.row_tiles;
    const int64_t rest = id / a.row_tiles;
    const int chunk = static_cast<int>(rest % a.chunks);
    const int head = static_cast<int>(rest / a.chunks % c.heads);
    const int64_t b = rest / a.chunks / c.heads;

    const int64_t rows = a.queries * a.group;
    const int64_t r0 = tile * kRows;
    const int64_t rl = r0 + kRows - 1 < rows - 1 ? r0 + kRows - 1 : rows - 1;      // last row
    const Row row = row_of(a, b, head, r0 + i16);
    // what the tile's rows see: from begin to at most stop, the row up to last
    const int64_t all = static_cast<int64_t>(a.s.pages_per_seq) << c.shift;
    int64_t begin = a.s.begin(b);
    begin = begin < 0 ? 0 : begin;
    const int64_t end = a.end ? a.end[b] : all;
    const int64_t row_end = end - (a.queries - 1 - (r0 + i16) / a.group);
    int64_t stop = end - (a.queries - 1 - rl / a.group);
    int64_t safe = end - (a.queries - 1 - r0 / a.group);        // every row sees up to here
    stop = stop > all ? all : stop;
    safe = safe > all ? all : safe;
    const int64_t base = begin & ~static_cast<int64_t>(kTile - 1);
    const int64_t c0 = base + chunk * a.chunk;
    const int64_t c1 = c0 + a.chunk < stop ? c0 + a.chunk : stop;
    if (a.part_o && c0 >= stop && chunk > 0) return;            // nothing there, and the join knows

    i32x4 qp[N][KK];
    const float unit = load_query<T, KK>(a, row, lane, qp);
    const float to_log2 = unit * a.scale * kLog2E;

    f32x4 o[JV];
#pragma unroll
    for (int j = 0; j < JV; j++) o[j] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    float step = 0x1p-126f, inv = 0x1p126f;                     // the running step of values

    const int block = static_cast<int>(c.block_bytes());
    const int64_t pitch = static_cast<int64_t>(c.heads) * 2 * block;
    const int8_t *data = c.data + static_cast<int64_t>(head) * 2 * block;
    const int32_t *table = a.s.table + b * a.s.table_stride;
    const int pmask = c.tokens() - 1;
    const int vcol = JV * i16 < c.width - JV ? JV * i16 : c.width - JV;

    for (int64_t t0 = c0 + wave * kTile; t0 < c1; t0 += NW * kTile) {
        // ---- where the tokens are ----
        int bad = 0;                                            // bit of a lane's 8 tokens: padding
        float ks[2][4], vs[2][4];
        i32x4 kv[2][KK];
        Columns<JV> vv[8];
        if constexpr (kWhole) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const int64_t t = t0 + 16 * u;
                int64_t page = -1;
                if (t < c1 && t + 16 > begin) page = table[t >> c.shift];
                const bool ok = page >= 0 && page < c.pages;
                const int64_t at = ok ? page : 0;
                const int8_t *kb = data + at * pitch;
                const int r = static_cast<int>(t) & pmask;
                const float2 sc = *reinterpret_cast<const float2 *>(c.scales + (at * c.heads + head) * 2);
#pragma unroll
                for (int kk = 0; kk < KK; kk++) {
                    const int col = 64 * kk + 16 * g < c.width - 16 ? 64 * kk + 16 * g : c.width - 16;
                    kv[u][kk] = *reinterpret_cast<const i32x4 *>(kb + (r + i16) * c.width + col);
                }
#pragma unroll
                for (int i = 0; i < 4; i++) vv[4 * u + i].load(kb + block + (r + 4 * g + i) * c.width + vcol);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    ks[u][i] = sc.x;
                    vs[u][i] = ok ? sc.y : 0.0f;
                }
                if (!ok) bad |= 0xf << (4 * u);
            }
        } else {
            const int64_t t = t0 + (lane & 31);
            int page = -1;
            if (t < c1 && t >= begin) page = table[t >> c.shift];
            const bool ok = page >= 0 && page < c.pages;
            page = ok ? page : 0;
            float2 sc = *reinterpret_cast<const float2 *>(c.scales + (static_cast<int64_t>(page) * c.heads + head) * 2);
            sc.y = ok ? sc.y : 0.0f;
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const int64_t at = __shfl(page, 16 * u + i16, kWave);
                const int8_t *kb = data + at * pitch + (static_cast<int>(t0 + 16 * u + i16) & pmask) * c.width;
#pragma unroll
                for (int kk = 0; kk < KK; kk++) {
                    const int col = 64 * kk + 16 * g < c.width - 16 ? 64 * kk + 16 * g : c.width - 16;
                    kv[u][kk] = *reinterpret_cast<const i32x4 *>(kb + col);
                }
            }
#pragma unroll
            for (int x = 0; x < 8; x++) {
                const int from = 16 * (x >> 2) + 4 * g + (x & 3);
                const int64_t at = __shfl(page, from, kWave);
                vv[x].load(data + at * pitch + block + (static_cast<int>(t0 + from) & pmask) * c.width + vcol);
                ks[x >> 2][x & 3] = __shfl(sc.x, from, kWave);
                vs[x >> 2][x & 3] = __shfl(sc.y, from, kWave);
                bad |= (__shfl(static_cast<int>(ok), from, kWave) ^ 1) << x;
            }
        }

        // ---- scores, in powers of two ----
        float s[2][4];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            i32x4 acc[N];
#pragma unroll
            for (int p = 0; p < N; p++) {
                acc[p] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < KK; kk++)
                    acc[p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kv[u][kk], qp[p][kk], acc[p], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float dot = static_cast<float>(acc[0][i] * 256 + acc[1][i]);
                if constexpr (N == 3) dot = __builtin_fmaf(dot, 256.0f, static_cast<float>(acc[2][i]));
                s[u][i] = dot * (ks[u][i] * to_log2);
            }
        }
        const bool inside = t0 >= begin && t0 + kTile <= safe;
        if (!inside || __ballot(bad) != 0) {
#pragma unroll
            for (int x = 0; x < 8; x++) {
                const int64_t t = t0 + 16 * (x >> 2) + 4 * g + (x & 3);
                if (t < begin || t >= row_end || t >= all) bad |= 1 << x;
                if ((bad >> x) & 1) s[x >> 2][x & 3] = -INFINITY;
            }
        }
        // ---- the running maximum and step ----
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                          fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        if (__ballot(top > m + kSlack<T>)) {
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float next = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - next);
            l *= f;
#pragma unroll
            for (int j = 0; j < JV; j++) o[j] *= f;
            m = next;
        }
        float big = fmaxf(fmaxf(fmaxf(vs[0][0], vs[0][1]), fmaxf(vs[0][2], vs[0][3])),
                          fmaxf(fmaxf(vs[1][0], vs[1][1]), fmaxf(vs[1][2], vs[1][3])));
        if (__ballot(big > 2.0f * step)) {
#pragma unroll
            for (int x = 1; x < kWave; x <<= 1) big = fmaxf(big, __shfl_xor(big, x, kWave));
            const float f = step / big;
#pragma unroll
            for (int j = 0; j < JV; j++) o[j] *= f;
            step = big;
            inv = 1.0f / big;
        }
        // ---- weights ----
        const float from = m == -INFINITY ? 0.0f : m - kOffset<T>;
        float w[8];
#pragma unroll
        for (int x = 0; x < 8; x++) {
            const float p = __builtin_amdgcn_exp2f(s[x >> 2][x & 3] - from);
            l += p;
            w[x] = (bad >> x) & 1 ? 0.0f : p * (vs[x >> 2][x & 3] * inv);
        }
        i32x4 hi, lo;
#pragma unroll
        for (int x = 0; x < 4; x++) {
            const int pair = pack_f16(w[2 * x], w[2 * x + 1]);
            hi[x] = pair;
            if constexpr (N == 3) {
                const f16x2 h = __builtin_bit_cast(f16x2, pair);    // of a scalar: hi[x] would be read as hi[0]
                lo[x] = pack_f16(w[2 * x] - static_cast<float>(h[0]), w[2 * x + 1] - static_cast<float>(h[1]));
            }
        }
        // ---- output ----
#pragma unroll
        for (int x = 0; x < 8; x++)
#pragma unroll
            for (int k = 0; k < Columns<JV>::kWords; k++) vv[x].w[k] ^= 0x80808080;
#pragma unroll
        for (int j = 0; j < JV; j++) {
            i32x4 v;
#pragma unroll
            for (int x = 0; x < 4; x++) v[x] = column_pair(vv[2 * x].w[j / 4], vv[2 * x + 1].w[j / 4], j % 4);
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, hi), o[j], 0, 0, 0);
            if constexpr (N == 3)
                o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, lo), o[j], 0, 0, 0);
        }
    }

    // ---- join the lanes of a row, then the wavefronts ----
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    const float back = step * 512.0f;
#pragma unroll
    for (int j = 0; j < JV; j++) o[j] *= back;
    if constexpr (NW > 1) {
        constexpr int kPad = 16 * JV + 4;
        __shared__ float so[NW - 1][kRows][kPad];
        __shared__ float sm[NW][kRows], sl[NW][kRows];
        if (lane < 16) {
            sm[wave][i16] = m;
            sl[wave][i16] = l;
        }
        if (wave > 0) {
#pragma unroll
            for (int j = 0; j < JV; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) so[wave - 1][i16][JV * (4 * g + i) + j] = o[j][i];
        }
        __syncthreads();
        if (wave > 0) return;
        float all_m = m;
#pragma unroll
        for (int x = 1; x < NW; x++) all_m = fmaxf(all_m, sm[x][i16]);
        const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - all_m);
        l *= f0;
#pragma unroll
        for (int j = 0; j < JV; j++) o[j] *= f0;
#pragma unroll
        for (int x = 1; x < NW; x++) {
            const float f = sm[x][i16] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[x][i16] - all_m);
            l += sl[x][i16] * f;
#pragma unroll
            for (int j = 0; j < JV; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) o[j][i] += so[x - 1][i16][JV * (4 * g + i) + j] * f;
        }
        m = all_m;
    }
    if (!row.there) return;
    if (a.part_o) {
        const int64_t r = ((b * c.heads + head) * rows + r0 + i16) * a.chunks + chunk;
        float *po = a.part_o + r * c.dim;
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int j = 0; j < JV; j++) {
                const int d = JV * (4 * g + i) + j;
                if (d < c.dim) po[d] = o[j][i];
            }
        if (g == 0) {
            a.part_ml[2 * r] = m;
            a.part_ml[2 * r + 1] = l;
        }
        return;
    }
    const bool none = m == -INFINITY;
    T *out = static_cast<T *>(a.out) + row.q * a.ot + row.head * a.oh;
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < JV; j++) {
            const int d = JV * (4 * g + i) + j;
            if (d < c.dim) out[d] = from_float<T>(none ? 0.0f : o[j][i] / l);
        }
    if (a.lse && g == 0)
        a.lse[row.q * (c.heads * a.group) + row.head] = none ? -INFINITY : (m - kOffset<T> + __builtin_amdgcn_logf(l)) / kLog2E;
}

// Joins the chunks of a row: a wavefront per row of a head.
template <class T>
__global__ __launch_bounds__(kBlock) void attend_join_kernel(const AttendArgs a) {
    const CacheView &c = a.c;
    const int lane = lane_id();
    const int64_t rows = a.queries * a.group;
    const int64_t all_rows = a.s.seqs * c.heads * rows;
    const int64_t x = static_cast<int64_t>(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave;
    if (x >= all_rows) return;
    const int64_t bh = x / rows, r = x - bh * rows;
    const int64_t b = bh / c.heads;
    const Row row = row_of(a, b, static_cast<int>(bh - b * c.heads), r);
    // the chunks that the row's tile has, as the tile counts them
    const int64_t rl = (r | (kRows - 1)) < rows - 1 ? (r | (kRows - 1)) : rows - 1;
    const int64_t all = static_cast<int64_t>(a.s.pages_per_seq) << c.shift;
    int64_t begin = a.s.begin(b);
    begin = begin < 0 ? 0 : begin;
    int64_t stop = (a.end ? a.end[b] : all) - (a.queries - 1 - rl / a.group);
    stop = stop > all ? all : stop;
    const int64_t span = stop - (begin & ~static_cast<int64_t>(kTile - 1));
    int64_t n = span <= 0 ? 1 : (span + a.chunk - 1) / a.chunk;
    n = n < a.chunks ? n : a.chunks;
    const float *ml = a.part_ml + 2 * x * a.chunks;
    const float *po = a.part_o + x * a.chunks * c.dim;
    float m = -INFINITY;
    for (int64_t i = lane; i < n; i += kWave) m = fmaxf(m, ml[2 * i]);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
    float l = 0.0f;
    float o[TGL_MAX_HEAD_DIM / kWave] = {};
    for (int64_t i0 = 0; i0 < n; i0 += kWave) {
        const int64_t i = i0 + lane;
        float f = 0.0f;
        if (i < n && ml[2 * i] != -INFINITY) f = __builtin_amdgcn_exp2f(ml[2 * i] - m);
        l += i < n ? ml[2 * i + 1] * f : 0.0f;
        const int count = n - i0 < kWave ? static_cast<int>(n - i0) : kWave;
        for (int y = 0; y < count; y++) {
            const float fy = __shfl(f, y, kWave);
#pragma unroll
            for (int k = 0; k < TGL_MAX_HEAD_DIM / kWave; k++)
                if (k * kWave + lane < c.dim) o[k] += po[(i0 + y) * c.dim + k * kWave + lane] * fy;
        }
    }
    l = group_sum<kWave>(l);
    const bool none = m == -INFINITY;
    T *out = static_cast<T *>(a.out) + row.q * a.ot + row.head * a.oh;
#pragma unroll
    for (int k = 0; k < TGL_MAX_HEAD_DIM / kWave; k++) {
        const int d = k * kWave + lane;
        if (d < c.dim) out[d] = from_float<T>(none ? 0.0f : o[k] / l);
    }
    if (a.lse && lane == 0)
        a.lse[row.q * (c.heads * a.group) + row.head] = none ? -INFINITY : (m - kOffset<T> + __builtin_amdgcn_logf(l)) / kLog2E;
}

// Workgroups that fill the card a few times over; a long axis is cut until
// there are that many, into chunks of at least kMinChunk tokens.
constexpr int64_t kFill = 2048;
constexpr int64_t kMinChunk = 256;

struct Plan {
    int64_t row_tiles;
    int64_t chunk;
    int32_t chunks;
    size_t part_o;          // bytes of each part of the workspace, 0 without chunks
    size_t part_ml;
};

Plan plan_of(const CacheView &c, int64_t num_seqs, int32_t pages_per_seq, int32_t q_heads, int64_t queries) {
    Plan p{};
    const int64_t rows = queries * (q_heads / c.heads);
    p.row_tiles = (rows + kRows - 1) / kRows;
    const int64_t most = (static_cast<int64_t>(pages_per_seq) << c.shift) + kTile;      // begin need not be at a step's start
    const int64_t items = num_seqs * c.heads * p.row_tiles;
    int64_t chunks = items > 0 ? kFill / items : 1;
    const int64_t cap = most / kMinChunk;
    chunks = chunks > cap ? cap : chunks;
    chunks = chunks < 1 ? 1 : chunks;
    p.chunk = (most + chunks - 1) / chunks;
    p.chunk = (p.chunk + 4 * kTile - 1) / (4 * kTile) * (4 * kTile);
    p.chunks = static_cast<int32_t>((most + p.chunk - 1) / p.chunk);
    if (p.chunks < 1) p.chunks = 1;
    if (p.chunks > 1) {
        const size_t n = static_cast<size_t>(num_seqs) * c.heads * rows * p.chunks;
        p.part_o = align_up(n * c.dim * 4, 256);
        p.part_ml = align_up(n * 8, 256);
    }
    return p;
}

template <class T, int JV, bool kWhole>
void launch(const AttendArgs &a, int nw, hipStream_t st) {
    const unsigned grid = static_cast<unsigned>((a.work + 7) / 8 * 8);
    if (nw == 1) attend_kernel<T, JV, kWhole, 1><<<grid, kWave, 0, st>>>(a);
    else attend_kernel<T, JV, kWhole, 4><<<grid, 4 * kWave, 0, st>>>(a);
}

template <class T>
void launch(const AttendArgs &a, int nw, hipStream_t st) {
    const bool whole = a.c.tokens() >= 16;
    if (a.c.width <= 32) whole ? launch<T, 2, true>(a, nw, st) : launch<T, 2, false>(a, nw, st);
    else if (a.c.width <= 64) whole ? launch<T, 4, true>(a, nw, st) : launch<T, 4, false>(a, nw, st);
    else if (a.c.width <= 128) whole ? launch<T, 8, true>(a, nw, st) : launch<T, 8, false>(a, nw, st);
    else whole ? launch<T, 16, true>(a, nw, st) : launch<T, 16, false>(a, nw, st);
    if (a.chunks > 1) {
        const int64_t rows = a.s.seqs * a.c.heads * a.queries * a.group;
        attend_join_kernel<T><<<static_cast<unsigned>((rows + 3) / 4), kBlock, 0, st>>>(a);
    }
}

// Rows without anything to see: zeros.
template <class T>
__global__ __launch_bounds__(kBlock) void attend_none_kernel(const AttendArgs a) {
    const int64_t rows = a.s.seqs * a.queries;
    const int heads = a.c.heads * a.group;
    const int64_t n = rows * heads * a.c.dim;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kBlock) {
        const int64_t rh = i / a.c.dim;
        static_cast<T *>(a.out)[rh / heads * a.ot + rh % heads * a.oh + i % a.c.dim] = from_float<T>(0.0f);
        if (a.lse && i % a.c.dim == 0) a.lse[rh] = -INFINITY;
    }
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

size_t tgl_cache_attend_workspace(const tgl_cache *cache, const tgl_seqs *seqs, int32_t q_heads, int64_t queries) {
    if (!valid_cache(cache) || !valid_seqs(seqs) || q_heads < 1 || q_heads > TGL_MAX_HEADS || q_heads % cache->heads != 0 ||
        queries < 1 || queries >= (int64_t(1) << 31))
        return 0;
    const Plan p = plan_of(view_of(*cache), seqs->num_seqs, seqs->pages_per_seq, q_heads, queries);
    return p.part_o + p.part_ml;
}

tgl_status tgl_cache_attend(const tgl_cache *cache, const tgl_heads *q, int32_t q_heads, int64_t queries,
                            int32_t dtype, const tgl_seqs *seqs, const int64_t *end, float scale,
                            const tgl_heads *out, float *lse, void *workspace, size_t workspace_bytes,
                            void *stream) {
    if (!valid_cache(cache) || !valid_seqs(seqs) || seqs->offsets || !is_elem_type(dtype)) return TGL_EINVAL;
    if (q_heads < 1 || q_heads > TGL_MAX_HEADS || q_heads % cache->heads != 0 || queries < 1) return TGL_EINVAL;
    if (queries >= (int64_t(1) << 31) || !aligned(end, 8) || !aligned(lse, 4) || !(scale == scale)) return TGL_EINVAL;
    const int64_t rows = seqs->num_seqs * queries;
    if (rows >= (int64_t(1) << 31) / q_heads) return TGL_EINVAL;
    if (!valid_heads(q, rows, dtype) || !valid_heads(out, rows, dtype)) return TGL_EINVAL;
    AttendArgs a{view_of(*cache), view_of(*seqs, rows), end, q->ptr, out->ptr, lse, nullptr, nullptr, q->token_stride,
                 q->head_stride, out->token_stride, out->head_stride, queries, 1, 0, 0, 1, q_heads / cache->heads, scale};
    const Plan p = plan_of(a.c, seqs->num_seqs, seqs->pages_per_seq, q_heads, queries);
    if (p.part_o + p.part_ml > 0) {
        if (!workspace || workspace_bytes < p.part_o + p.part_ml) return TGL_ENOSPACE;
        if (!aligned(workspace, 256)) return TGL_EINVAL;
    }
    if (rows == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (cache->num_pages == 0 || seqs->pages_per_seq == 0) {
        const int64_t n = (rows * q_heads * a.c.dim + kBlock - 1) / kBlock;
        const unsigned grid = static_cast<unsigned>(n < (1 << 16) ? n : 1 << 16);
        if (dtype == TGL_OUT_F32) attend_none_kernel<float><<<grid, kBlock, 0, st>>>(a);
        else attend_none_kernel<bf16_t><<<grid, kBlock, 0, st>>>(a);
        return launch_status();
    }
    a.row_tiles = p.row_tiles;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.work = seqs->num_seqs * a.c.heads * p.row_tiles * p.chunks;
    if (a.work > 0x7ffffff0) return TGL_EINVAL;
    if (p.part_o) {
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part_o);
    }
    // a wavefront alone where a sequence has at most two steps for it
    const int nw = (static_cast<int64_t>(a.s.pages_per_seq) << a.c.shift) <= 2 * kTile ? 1 : 4;
    if (dtype == TGL_OUT_F32) launch<float>(a, nw, st);
    else launch<bf16_t>(a, nw, st);
    return launch_status();
}

}  // extern "C"
