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
//           they lie in the cache; a query row goes in as three signed bytes of
//           a 24-bit whole number, in units of its largest element / (127 *
//           65536).  The sums are exact; what is lost is that rounding, 2^-24
//           of the row's largest element.  (Two bytes would do for the large
//           elements of a bfloat16 row, but one outlier among them would take
//           the others' bits.)
//   output  O^T = V^T P^T on the f16 ones.  S^T leaves every lane four tokens
//           of a row per 16 x 16 tile, which is what P^T takes with the tokens
//           in a fixed other order, so the probabilities never leave their
//           lane.  V^T wants, per lane, one column of eight tokens: a lane
//           loads the same few columns of its eight tokens and picks a
//           column's bytes with v_perm.  A byte b ^ 0x80 = v + 128 read as the bits
//           of an f16 is (v + 128) 2^-24, and one packed fused multiply-add
//           makes it v 2^-9, exactly.
//   P       carries the step of its token's page.  Its unit is a row's own: a
//           power of two that follows the largest exponential times step that
//           the row has summed, so that what has weight keeps its bits, however
//           large the steps are of what has none or is not seen.  P is two f16,
//           the second the rounding error of the first: 2^-22 of each weight,
//           or 2^-36 of the largest.
//
// Few rows a head: bound by memory.  1,000,003 tokens of 8 heads of 128 in pages
// of 64 (2.05 GB), 4 query heads each, 350 us, 5.9 TB/s, and 8 us to join 253
// chunks; 64 histories of 1 to 8192 tokens (0.54 GB) 114 + 5 us, 4.5 TB/s, the
// rest being long and short histories side by side; float32 queries the same.
// Small pages and heads: half by instructions, 330 for 32 tokens, half by the
// latency of rows that are not loaded a step ahead (600 windows of 1000 tokens,
// 2 heads of 64, pages of 4: 37 us, 3.5 TB/s).  Many rows: by the scores'
// arithmetic (256 queries of 4 histories of 2500 to 4097, 8 heads of 128 for 32:
// 130 us, 410 TFLOP/s), 460 vector instructions for 32 rows and 32 tokens beside
// 56 matrix ones.  (With a query in two bytes and P in one f16: 95 us, and
// outputs that are off by that rounding.)
#include "tgl_cache.hpp"

namespace tgl {
namespace {

using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

constexpr int kRows = 16;           // rows of a tile
constexpr int kTile = 32;           // tokens of a wavefront's step
constexpr float kLowest = -3.4028235e38f;
constexpr float kLog2E = 1.44269504088896340736f;

enum Order { kInTurn, kHeadsInTurn, kStretches };

struct AttendArgs {
    CacheView c;
    SeqsView s;
    const int64_t *end;
    const void *q;
    void *out;
    float *lse;
    float *part_o;          // [rows of all heads][chunks][width], or null
    float *part_ml;         // [rows of all heads][chunks][2]
    int64_t qt, qh, ot, oh;
    int64_t chunk;          // tokens of a workgroup, below 2^31
    uint32_t queries;
    uint32_t rows;          // of one sequence and head: queries * group
    uint32_t work;          // workgroups
    uint32_t chunks;
    uint32_t tile_rows;     // rows of a workgroup: 16, or 32
    uint32_t all_rows;      // rows of all sequences and heads
    Div tiles;              // row tiles of one sequence and head
    Div items;              // sequences times heads
    Div heads;
    Div group;              // query heads of one head of the cache
    Div row_of;             // rows of one sequence and head
    int32_t order;          // of the workgroups: see die_order
    float scale;
};

// The unit of work of a workgroup: a row tile, fastest, of a sequence's head's
// chunk.  Workgroups go to the 8 dies in turn.  Row tiles of one head read the
// same tokens, so all of them go to one die, whose L2 then serves them: heads
// in turn (the dies get long and short sequences alike), or, where that would
// leave dies with less, a contiguous stretch of the work each.
__device__ __forceinline__ uint32_t die_order(const AttendArgs &a) {
    if (a.order == kInTurn) return blockIdx.x;
    const uint32_t die = blockIdx.x & 7, at = blockIdx.x >> 3;
    if (a.order == kHeadsInTurn) {
        const uint32_t head = a.tiles(at);
        return (head * 8 + die) * a.tiles.d + (at - head * a.tiles.d);      // beyond the work for the last heads
    }
    const uint32_t per = (a.work + 7) / 8;
    return at >= per ? a.work : die * per + at;
}

constexpr int kParts = 3;           // bytes of a query element

// Exponentials are taken relative to a whole power of two, which is raised when
// one of them would pass 2^kSlack: their sum is float32 and has room.
constexpr float kSlack = 4.0f;

// Exponential times step in the row's unit is f16.  One that would pass kLimit
// makes the unit larger, so that it lies in [2^(kTop - 1), 2^kTop).  kFinest is the
// inverse of the smallest unit, which is the first: steps are at least 2^-107.
constexpr float kLimit = 32768.0f, kFinest = 0x1p126f;
constexpr int kTop = 12;

// The row's query as signed bytes, kk-th piece of 64 columns, part p (the
// highest first); returns the size of one unit.  v + 0x808080 has, byte by
// byte, the digits of v in base 256 between -128 and 127, each plus 128.
template <class T, int KK>
__device__ __forceinline__ float load_query(const AttendArgs &a, const T *q, bool there, int lane, i32x4 (&parts)[kParts][KK]) {
    float x[KK][16];
    uint32_t bits = 0;              // of the largest magnitude: NaN above infinity above numbers
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
        load_columns<T, 16>(q, 64 * kk + 16 * (lane >> 4), a.c.dim, x[kk]);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const uint32_t v = __builtin_bit_cast(uint32_t, x[kk][i]) & 0x7fffffffu;
            bits = v > bits ? v : bits;
        }
    }
    uint32_t other = __shfl_xor(bits, 16, kWave);
    bits = other > bits ? other : bits;
    other = __shfl_xor(bits, 32, kWave);
    bits = other > bits ? other : bits;
    const float top = __builtin_bit_cast(float, bits);
    constexpr float kUnits = 127.0f * 65536.0f;
    // not finite: a NaN unit makes the row NaN; tiny: zeros
    const float unit = bits >= 0x7f800000u ? __builtin_nanf("") : top < kTiny ? 0.0f : top * (1.0f / kUnits);
    const float size = there ? inverse_step(unit) : 0.0f;
    const float inv = a.scale < 0.0f ? -size : size;     // the sign of the scale goes into the bytes
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
#pragma unroll
        for (int w = 0; w < 4; w++) {
            int v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float y = inv == 0.0f ? 0.0f : x[kk][4 * w + i] * inv;
                v[i] = static_cast<int>(rintf(y)) + 0x808080;
            }
#pragma unroll
            for (int p = 0; p < kParts; p++) {
                const unsigned byte = kParts - 1 - p;
                const unsigned two = 0x0c0c0000u | ((4 + byte) << 8) | byte;
                const int ab = __builtin_amdgcn_perm(v[1], v[0], two), cd = __builtin_amdgcn_perm(v[3], v[2], two);
                parts[p][kk][w] = (ab | (cd << 16)) ^ 0x80808080;
            }
        }
    }
    return unit;
}

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

// The value, as if computed here: an address made of a uniform pointer and a
// 32-bit offset of the lane is one operand each only where the compiler sees
// that the offset has 32 bits, not where it has moved that out of a loop over t.
__device__ __forceinline__ uint32_t here(uint32_t v, int t) {
    asm("" : "+v"(v) : "s"(t));
    return v;
}

// What the queries of a sequence see, whatever the device arrays say: begin in
// [0, all], the end of the last query's view in [0, all + queries].
struct View {
    int64_t begin, end, all;
};

__device__ __forceinline__ View view_of_seq(const AttendArgs &a, uint32_t b) {
    View v;
    v.all = static_cast<int64_t>(a.s.pages_per_seq) << a.c.shift;
    v.begin = a.s.begin(b);
    v.begin = v.begin < 0 ? 0 : v.begin > v.all ? v.all : v.begin;
    v.end = a.end ? a.end[b] : v.all;
    const int64_t most = v.all + a.queries;
    v.end = v.end < 0 ? 0 : v.end > most ? most : v.end;
    return v;
}

__device__ __forceinline__ int clamp_to(int64_t v, int most) {
    return v < 0 ? 0 : v > most ? most : static_cast<int>(v);
}

// What of a wavefront's 32 tokens is surely on one page: a token (pages of 1 and
// 2), the four that a lane has of each half (4 and 8), a half (16 and more).
enum Pages { kTokens, kFours, kHalves };

// Wavefronts of a SIMD that the registers are cut for: the most that spill
// nothing, or (pages of 1 and 2, heads above 32) a few.
template <int JV, int R>
constexpr int kWavesPerSimd = JV >= 8 || R == 2 ? 2 : 4;

// A wavefront's 32 tokens: where they are, then what they hold.
template <int JV, int kPages>
struct Step {
    static constexpr int KK = JV >= 4 ? JV / 4 : 1;
    static constexpr int kLooks = kPages == kHalves ? 2 : 1;
    int page[kLooks];               // kHalves: of the two, uniform; else of token lane & 31; -1: nothing to see
    float2 sc[kLooks];              // the steps of keys and values
    i32x4 kv[2][KK];
    Columns<JV> vv[8];
};

// JV: columns of a lane, so heads of up to 16 JV.  kPages: see Pages.  NW:
// wavefronts that share a workgroup's tokens.  R: row tiles of a wavefront, which share the keys'
// loads and the values' conversion.
template <class T, int JV, int kPages, int NW, int R>
__global__ __launch_bounds__(NW * kWave, (kWavesPerSimd<JV, R>)) void attend_kernel(const AttendArgs a) {
    constexpr int KK = JV >= 4 ? JV / 4 : 1;
    constexpr bool kWhole = kPages == kHalves;
    constexpr int kLooks = Step<JV, kPages>::kLooks;
    const CacheView &c = a.c;
    const int lane = lane_id();
    const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int g = lane >> 4, i16 = lane & 15;
    const uint32_t id = die_order(a);
    if (id >= a.work) return;
    // row tiles first, then heads and sequences, chunks last: the chunks that
    // only long sequences have are then spread over the dies
    const uint32_t rest = a.tiles(id);
    const uint32_t tile = id - rest * a.tiles.d;
    const uint32_t chunk = a.items(rest);
    const uint32_t bh = rest - chunk * a.items.d;                       // sequence and head
    const uint32_t b = a.heads(bh);
    const int head = static_cast<int>(bh - b * a.heads.d);

    const uint32_t r0 = tile * (kRows * R);
    const uint32_t rl = r0 + kRows * R < a.rows ? r0 + kRows * R - 1 : a.rows - 1;      // last row
    // what the tile's rows see: from begin to at most stop, a row up to row_end
    const View view = view_of_seq(a, b);
    const int64_t all = view.all, begin = view.begin, end = view.end;
    int64_t stop = end - (a.queries - 1 - a.group(rl));
    int64_t safe = end - (a.queries - 1 - a.group(r0));                 // every row sees up to here
    stop = stop > all ? all : stop;
    safe = safe > all ? all : safe;
    const int64_t c0 = (begin & ~static_cast<int64_t>(kTile - 1)) + chunk * a.chunk;
    if (a.part_o && c0 >= stop && chunk > 0) return;            // nothing there, and the join knows
    // positions from here on count from c0
    const int n = clamp_to(stop - c0, static_cast<int>(a.chunk));
    const int first = clamp_to(begin - c0, n), full = clamp_to(safe - c0, n);

    bool there[R];
    int64_t q_row[R];
    int q_head[R], last[R];
    i32x4 qp[R][kParts][KK];
    float to_log2[R];
#pragma unroll
    for (int y = 0; y < R; y++) {
        const uint32_t at = r0 + kRows * y + i16;
        there[y] = at < a.rows;
        const uint32_t r = there[y] ? at : rl;
        const uint32_t t = a.group(r);                                  // the lane's query
        q_row[y] = static_cast<int64_t>(b) * a.queries + t;
        q_head[y] = static_cast<int>(head * a.group.d + (r - t * a.group.d));
        int64_t row_end = end - (a.queries - 1 - t);
        row_end = row_end > all ? all : row_end;
        last[y] = clamp_to(row_end - c0, n);
        const float unit = load_query<T, KK>(a, static_cast<const T *>(a.q) + q_row[y] * a.qt + q_head[y] * a.qh, there[y], lane, qp[y]);
        to_log2[y] = unit * fabsf(a.scale) * kLog2E;
    }

    f32x4 o[R][JV];
    float m[R], l[R], inv[R];                                   // inv: of the unit that o is in, 2^-9 of it
    int unseen[R];                                              // bit k: none of the lane's k-th tokens was seen
#pragma unroll
    for (int y = 0; y < R; y++) {
        m[y] = -INFINITY;
        l[y] = 0.0f;
        inv[y] = kFinest;
        unseen[y] = 0xff;
#pragma unroll
        for (int j = 0; j < JV; j++) o[y][j] = f32x4{0, 0, 0, 0};
    }

    const uint32_t width = c.width;
    const uint32_t block = width << c.shift;
    const uint32_t pitch = a.heads.d * 2 * block;
    const int8_t *data = c.data + static_cast<int64_t>(head) * 2 * block;
    const float2 *steps = reinterpret_cast<const float2 *>(c.scales) + head;
    const uint32_t pages = static_cast<uint32_t>(c.pages);
    const uint32_t pmask = c.tokens() - 1;
    const int32_t *table = a.s.table + b * a.s.table_stride + (c0 >> c.shift);
    const uint32_t c0r = static_cast<uint32_t>(c0) & pmask;     // c0's row in its page
    // a lane's columns: those of a row that lie beyond its width are read from its end and not used
    uint32_t kcol[KK];
#pragma unroll
    for (int kk = 0; kk < KK; kk++) kcol[kk] = 64 * kk + 16 * g < static_cast<int>(width) - 16 ? 64 * kk + 16 * g : width - 16;
    const uint32_t vcol = JV * i16 < static_cast<int>(width) - JV ? JV * i16 : width - JV;

    uint32_t kat[KK], vat[4];                                   // places in a half step whose rows are one after another
#pragma unroll
    for (int kk = 0; kk < KK; kk++) kat[kk] = i16 * width + kcol[kk];
#pragma unroll
    for (int i = 0; i < 4; i++) vat[i] = (4 * g + i) * width + vcol;

    // the pages of the step at t0 (whose table entries exist up to token n - 1)
    auto look_up = [&](int t0, int (&page)[kLooks]) {
        if constexpr (kWhole) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const int p = t0 + 16 * u;
                const int got = table[(c0r + (p < n ? p : n - 1)) >> c.shift];
                page[u] = p < n && p + 16 > first && static_cast<uint32_t>(got) < pages ? got : -1;
            }
        } else {
            // kFours: as far as one of the four is seen
            const int p = t0 + (lane & 31), from = kPages == kFours ? p & ~3 : p, to = kPages == kFours ? p | 3 : p;
            const int got = table[(c0r + (from < n ? from : n - 1)) >> c.shift];
            page[0] = from < n && to >= first && static_cast<uint32_t>(got) < pages ? got : -1;
        }
    };

    // the rows and steps of the step at t0, whose pages are known
    auto fetch = [&](int t0, Step<JV, kPages> &x) {
        if constexpr (kWhole) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const uint32_t at = x.page[u] < 0 ? 0 : x.page[u];
                x.sc[u] = steps[static_cast<uint64_t>(at) * a.heads.d];
                const int8_t *kb = data + static_cast<uint64_t>(at) * pitch + ((c0r + t0 + 16 * u) & pmask) * width;
#pragma unroll
                for (int kk = 0; kk < KK; kk++) x.kv[u][kk] = *reinterpret_cast<const i32x4 *>(kb + here(kat[kk], t0));
                const int8_t *vb = kb + block;
#pragma unroll
                for (int i = 0; i < 4; i++) x.vv[4 * u + i].load(vb + here(vat[i], t0));
            }
        } else {
            const uint32_t own = x.page[0] < 0 ? 0 : x.page[0];
            x.sc[0] = steps[static_cast<uint64_t>(own) * a.heads.d];
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const uint32_t at = __builtin_amdgcn_ds_bpermute(4 * (16 * u + i16), own);
                const int8_t *kb = data + static_cast<uint64_t>(at) * pitch + ((c0r + t0 + 16 * u + i16) & pmask) * width;
#pragma unroll
                for (int kk = 0; kk < KK; kk++) x.kv[u][kk] = *reinterpret_cast<const i32x4 *>(kb + kcol[kk]);
            }
            if constexpr (kPages == kFours) {
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    const int from = 16 * u + 4 * g;
                    const uint32_t at = __builtin_amdgcn_ds_bpermute(4 * from, own);
                    const int8_t *vb = data + static_cast<uint64_t>(at) * pitch + block + ((c0r + t0 + from) & pmask) * width + vcol;
#pragma unroll
                    for (int i = 0; i < 4; i++) x.vv[4 * u + i].load(vb + i * width);
                }
            }
#pragma unroll
            for (int k = 0; k < (kPages == kTokens ? 8 : 0); k++) {
                const int from = 16 * (k >> 2) + 4 * g + (k & 3);
                const uint32_t at = __builtin_amdgcn_ds_bpermute(4 * from, own);
                x.vv[k].load(data + static_cast<uint64_t>(at) * pitch + block + ((c0r + t0 + from) & pmask) * width + vcol);
            }
        }
    };

    auto multiply = [&](int t0, Step<JV, kPages> &x) {
        // ---- steps of the lane's 8 tokens, which of them nobody sees ----
        int bad = 0;
        float ks[8], vs[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            if constexpr (kWhole) {
                const bool ok = x.page[k >> 2] >= 0;
                ks[k] = x.sc[k >> 2].x;
                vs[k] = ok ? x.sc[k >> 2].y : 0.0f;
                if (!ok) bad |= 1 << k;
            } else if (kPages == kFours && (k & 3) != 0) {
                ks[k] = ks[k & ~3];
                vs[k] = vs[k & ~3];
                bad |= ((bad >> (k & ~3)) & 1) << k;
            } else {
                const int from = 4 * (16 * (k >> 2) + 4 * g + (k & 3));
                const float y = x.page[0] < 0 ? 0.0f : x.sc[0].y;
                ks[k] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(from, __builtin_bit_cast(int, x.sc[0].x)));
                vs[k] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(from, __builtin_bit_cast(int, y)));
                bad |= (__builtin_amdgcn_ds_bpermute(from, x.page[0]) < 0 ? 1 : 0) << k;
            }
        }
        const bool inside = t0 >= first && t0 + kTile <= full;
        bool masked = !inside;
        if constexpr (kWhole) masked = masked || x.page[0] < 0 || x.page[1] < 0;
        else masked = masked || __ballot(x.page[0] < 0) != 0;

        i32x4 hi[R], lo[R];
#pragma unroll
        for (int y = 0; y < R; y++) {
            // ---- dots; a score, in powers of two, is dot * unit, unit >= 0 ----
            float dot[8], unit[8];
#pragma unroll
            for (int u = 0; u < 2; u++) {
                i32x4 acc[kParts];
#pragma unroll
                for (int p = 0; p < kParts; p++) {
                    acc[p] = i32x4{0, 0, 0, 0};
#pragma unroll
                    for (int kk = 0; kk < KK; kk++)
                        acc[p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x.kv[u][kk], qp[y][p][kk], acc[p], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    dot[4 * u + i] = __builtin_fmaf(static_cast<float>(acc[0][i] * 256 + acc[1][i]), 256.0f, static_cast<float>(acc[2][i]));
                    unit[4 * u + i] = ks[4 * u + i] * to_log2[y];
                }
            }
            const float unit0 = unit[0], unit4 = unit[4];
            int hide = bad;
            if (masked) {
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    const int p = t0 + 16 * (k >> 2) + 4 * g + (k & 3);
                    if (p < first || p >= last[y]) hide |= 1 << k;
                    const bool hidden = (hide >> k) & 1;
                    dot[k] = hidden ? -INFINITY : dot[k];
                    unit[k] = hidden ? 1.0f : unit[k];          // -inf stays -inf whatever the page's step is
                }
            }
            unseen[y] &= hide;
            // ---- the running maximum (of nothing where -inf meets a unit of 0: NaN, which fmaxf drops) ----
            float top;
            if constexpr (kPages != kTokens) {                  // one unit for each half's four
                top = fmaxf(fmaxf(fmaxf(dot[0], dot[1]), fmaxf(dot[2], dot[3])) * unit0,
                            fmaxf(fmaxf(dot[4], dot[5]), fmaxf(dot[6], dot[7])) * unit4);
            } else {
                top = dot[0] * unit[0];
#pragma unroll
                for (int k = 1; k < 8; k++) top = fmaxf(top, dot[k] * unit[k]);
            }
            if (__ballot(top > m[y] + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16, kWave));
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float next = fmaxf(m[y], ceilf(top));
                if (m[y] != -INFINITY) {
                    // o stays as it is: relative to the new maximum its unit is smaller
                    const float finer = inv[y] * __builtin_amdgcn_exp2f(next - m[y]);
                    l[y] *= __builtin_amdgcn_exp2f(m[y] - next);
                    inv[y] = finer > kFinest ? kFinest : finer;
                    if (finer > kFinest) {
#pragma unroll
                        for (int j = 0; j < JV; j++) o[y][j] *= kFinest / finer;
                    }
                }
                m[y] = next;
            }
            // ---- weights, times steps ----
            const float from = m[y] == -INFINITY ? 0.0f : m[y];
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(dot[k], unit[k], -from));
                l[y] += p;
                w[k] = p * vs[k];
            }
            if (masked) {
#pragma unroll
                for (int k = 0; k < 8; k++) w[k] = (hide >> k) & 1 ? 0.0f : w[k];    // a step that is not seen may be NaN
            }
            // ---- the row's unit ----
            float big = fmaxf(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7])));
            if (__ballot(big * inv[y] > kLimit)) {
                big = fmaxf(big, __shfl_xor(big, 16, kWave));
                big = fmaxf(big, __shfl_xor(big, 32, kWave));
                if (big * inv[y] > kLimit) {
                    const float next = ldexpf(1.0f, kTop - __builtin_amdgcn_frexp_expf(big));
#pragma unroll
                    for (int j = 0; j < JV; j++) o[y][j] *= next / inv[y];
                    inv[y] = next;
                }
            }
#pragma unroll
            for (int k = 0; k < 8; k++) w[k] *= inv[y];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                int pair = pack_f16(w[2 * k], w[2 * k + 1]);
                asm("" : "+v"(pair));                                   // or each half would be converted once more by itself
                hi[y][k] = pair;
                const f16x2 h = __builtin_bit_cast(f16x2, pair);        // of a scalar: hi[y][k] would be read as hi[y][0]
                lo[y][k] = pack_f16(__builtin_fmaf(static_cast<float>(h[0]), -1.0f, w[2 * k]),
                                    __builtin_fmaf(static_cast<float>(h[1]), -1.0f, w[2 * k + 1]));
            }
        }
        // ---- output ----
#pragma unroll
        for (int k = 0; k < 8; k++)
#pragma unroll
            for (int w = 0; w < Columns<JV>::kWords; w++) x.vv[k].w[w] ^= 0x80808080;
#pragma unroll
        for (int j = 0; j < JV; j++) {
            i32x4 v;
#pragma unroll
            for (int k = 0; k < 4; k++) v[k] = column_pair(x.vv[2 * k].w[j / 4], x.vv[2 * k + 1].w[j / 4], j % 4);
#pragma unroll
            for (int y = 0; y < R; y++) {
                o[y][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, hi[y]), o[y][j], 0, 0, 0);
                o[y][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, lo[y]), o[y][j], 0, 0, 0);
            }
        }
    };

    constexpr int kNext = NW * kTile;
    constexpr bool kAhead = kWhole && JV < 16 && !(JV == 8 && R == 2);      // as far as registers go
    int t0 = wave * kTile;
    if (t0 < n) {
        if constexpr (!kAhead) {
            // the next step's pages are looked up while this one's rows come;
            // other wavefronts hide the rows' latency
            Step<JV, kPages> x;
            look_up(t0, x.page);
            for (; t0 < n; t0 += kNext) {
                fetch(t0, x);
                int page[kLooks];
                look_up(t0 + kNext, page);
                __builtin_amdgcn_sched_barrier(0);
                multiply(t0, x);
#pragma unroll
                for (int u = 0; u < kLooks; u++) x.page[u] = page[u];
            }
        } else {
            // two wavefronts a SIMD hide little: rows come a step ahead, too
            Step<JV, kPages> x, y;
            look_up(t0, x.page);
            fetch(t0, x);
            look_up(t0 + kNext, y.page);
            for (; t0 < n; t0 += 2 * kNext) {
                fetch(t0 + kNext, y);
                int page[kLooks];
                look_up(t0 + 2 * kNext, page);
                __builtin_amdgcn_sched_barrier(0);
                multiply(t0, x);
#pragma unroll
                for (int u = 0; u < kLooks; u++) x.page[u] = page[u];
                if (t0 + kNext >= n) break;
                fetch(t0 + 2 * kNext, x);
                look_up(t0 + 3 * kNext, page);
                __builtin_amdgcn_sched_barrier(0);
                multiply(t0 + kNext, y);
#pragma unroll
                for (int u = 0; u < kLooks; u++) y.page[u] = page[u];
            }
        }
    }

    // ---- join the lanes of a row, then the wavefronts ----
    // what is joined is means, with weights of at most 1: sums of values could overflow
    constexpr int kPad = 16 * JV + 4;
    __shared__ float so[NW > 1 ? NW - 1 : 1][kRows][kPad];
    __shared__ float sm[NW][kRows], sl[NW][kRows];
#pragma unroll
    for (int y = 0; y < R; y++) {
        l[y] += __shfl_xor(l[y], 16, kWave);
        l[y] += __shfl_xor(l[y], 32, kWave);
        // -inf is the maximum of nothing; seen scores of -inf have a maximum below every other
        const bool seen = __shfl_xor(unseen[y], 16, kWave) != 0xff || __shfl_xor(unseen[y], 32, kWave) != 0xff ||
                          __shfl_xor(unseen[y], 48, kWave) != 0xff || unseen[y] != 0xff;
        if (m[y] == -INFINITY && seen) m[y] = kLowest;
        const float back = 512.0f / inv[y];
        float norm = l[y] == 0.0f ? 0.0f : back / l[y];         // a NaN among what is seen stays one
        if constexpr (NW > 1) {
            if (y > 0) __syncthreads();
            if (lane < 16) {
                sm[wave][i16] = m[y];
                sl[wave][i16] = l[y];
            }
            if (wave > 0) {
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < JV; j++) so[wave - 1][i16][JV * (4 * g + i) + j] = o[y][j][i] * norm;
            }
            __syncthreads();
            if (wave == 0) {
                float all_m = m[y];
#pragma unroll
                for (int w = 1; w < NW; w++) all_m = fmaxf(all_m, sm[w][i16]);
                float f[NW];
                f[0] = m[y] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[y] - all_m);
                l[y] *= f[0];
#pragma unroll
                for (int w = 1; w < NW; w++) {
                    f[w] = sl[w][i16] * (sm[w][i16] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[w][i16] - all_m));
                    l[y] += f[w];
                }
                const float part = l[y] == 0.0f ? 0.0f : 1.0f / l[y];
#pragma unroll
                for (int j = 0; j < JV; j++) o[y][j] *= back * (f[0] * part);
#pragma unroll
                for (int w = 1; w < NW; w++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
#pragma unroll
                        for (int j = 0; j < JV; j++) o[y][j][i] += so[w - 1][i16][JV * (4 * g + i) + j] * (f[w] * part);
                m[y] = all_m;
                norm = 1.0f;
            }
        }
        const bool none = m[y] == -INFINITY;
        if (wave == 0 && there[y] && a.part_o) {
            const int64_t at = (static_cast<int64_t>(bh) * a.rows + r0 + kRows * y + i16) * a.chunks + chunk;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float v[JV];
#pragma unroll
                for (int j = 0; j < JV; j++) v[j] = o[y][j][i] * norm;
                store_columns<float, JV>(a.part_o + at * width, JV * (4 * g + i), width, v);
            }
            if (g == 0) {
                a.part_ml[2 * at] = m[y];
                a.part_ml[2 * at + 1] = l[y];
            }
        }
        if (wave == 0 && there[y] && !a.part_o) {
            if (!none && l[y] == 0.0f) l[y] = norm = __builtin_nanf("");    // the largest score is infinite
            T *out = static_cast<T *>(a.out) + q_row[y] * a.ot + q_head[y] * a.oh;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float v[JV];
#pragma unroll
                for (int j = 0; j < JV; j++) v[j] = none ? 0.0f : o[y][j][i] * norm;
                store_columns<T, JV>(out, JV * (4 * g + i), c.dim, v);
            }
            if (a.lse && g == 0)
                a.lse[q_row[y] * (a.heads.d * a.group.d) + q_head[y]] = none ? -INFINITY : (m[y] + __builtin_amdgcn_logf(l[y])) / kLog2E;
        }
    }
}

// Joins the chunks of a row, a mean each, with NW wavefronts.  A lane takes four columns of
// every (NW kWave / kLanes)-th chunk, kLanes the lanes of a row's columns, eight
// chunks in flight (253 chunks of 32 rows of 128: 8 us; 212 us with a wavefront
// per row and a chunk at a time).  With NW = 1 a workgroup has a row for each of its
// wavefronts.
template <class T, int NW, int kLanes>
__global__ __launch_bounds__((NW == 1 ? kBlock : NW * kWave)) void attend_join_kernel(const AttendArgs a) {
    constexpr int kStep = 8, kStride = NW * kWave / kLanes;
    __shared__ float so[NW][4 * kLanes];
    __shared__ float sl[NW], sm[NW];
    const CacheView &c = a.c;
    const int lane = lane_id();
    const int at_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wave = NW == 1 ? 0 : at_wave;
    const uint32_t x = NW == 1 ? blockIdx.x * (kBlock / kWave) + at_wave : blockIdx.x;
    if (NW == 1 && x >= a.all_rows) return;
    const uint32_t bh = a.row_of(x), r = x - bh * a.rows;
    const uint32_t b = a.heads(bh), t = a.group(r);
    const int64_t q_row = static_cast<int64_t>(b) * a.queries + t;
    const int q_head = static_cast<int>((bh - b * a.heads.d) * a.group.d + (r - t * a.group.d));
    // the chunks that the row's tile has, as the tile counts them
    const uint32_t tile_end = r / a.tile_rows * a.tile_rows + a.tile_rows;
    const uint32_t rl = tile_end < a.rows ? tile_end - 1 : a.rows - 1;
    const View view = view_of_seq(a, b);
    int64_t stop = view.end - (a.queries - 1 - a.group(rl));
    stop = stop > view.all ? view.all : stop;
    const int64_t span = stop - (view.begin & ~static_cast<int64_t>(kTile - 1));
    const int64_t want = span <= 0 ? 1 : (span + a.chunk - 1) / a.chunk;
    const int n = static_cast<int>(want < a.chunks ? want : a.chunks);
    const int64_t at = (static_cast<int64_t>(bh) * a.rows + r) * a.chunks;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + at;
    const int col = 4 * (lane % kLanes) < c.width ? 4 * (lane % kLanes) : 0;
    const float *po = a.part_o + at * c.width + col;
    float m = -INFINITY;
    for (int i = wave * kWave + lane; i < n; i += NW * kWave) m = fmaxf(m, ml[i].x);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
    if constexpr (NW > 1) {
        if (lane == 0) sm[wave] = m;
        __syncthreads();
#pragma unroll
        for (int y = 0; y < NW; y++) m = fmaxf(m, sm[y]);
    }
    float l = 0.0f;
    for (int i = wave * kWave + lane; i < n; i += NW * kWave) {
        const float2 w = ml[i];
        l += w.y * (w.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(w.x - m));
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) l += __shfl_xor(l, d, kWave);
    if constexpr (NW > 1) {
        if (lane == 0) sl[wave] = l;
        __syncthreads();
        l = 0.0f;
#pragma unroll
        for (int y = 0; y < NW; y++) l += sl[y];
    }
    const bool none = m == -INFINITY;
    if (!none && l == 0.0f) l = __builtin_nanf("");         // the largest score is infinite
    const float part = none ? 0.0f : 1.0f / l;
    f32x4 o = {0, 0, 0, 0};
    for (int i0 = (wave * kWave + lane) / kLanes; i0 < n; i0 += kStep * kStride) {
        f32x4 v[kStep];
        float2 w[kStep];
#pragma unroll
        for (int y = 0; y < kStep; y++) {
            const int i = i0 + y * kStride < n ? i0 + y * kStride : n - 1;
            w[y] = ml[i];
            v[y] = *reinterpret_cast<const f32x4 *>(po + static_cast<int64_t>(i) * c.width);
        }
#pragma unroll
        for (int y = 0; y < kStep; y++) {
            if (i0 + y * kStride >= n) continue;
            o += v[y] * (w[y].y * (w[y].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(w[y].x - m)) * part);
        }
    }
    // the wavefront's other chunks, then the other wavefronts
#pragma unroll
    for (int d = kLanes; d < kWave; d <<= 1)
#pragma unroll
        for (int k = 0; k < 4; k++) o[k] += __shfl_xor(o[k], d, kWave);
    if constexpr (NW > 1) {
        if (lane < kLanes) *reinterpret_cast<f32x4 *>(&so[wave][4 * lane]) = o;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int y = 1; y < NW; y++) o += *reinterpret_cast<const f32x4 *>(&so[y][4 * (lane % kLanes)]);
    }
    T *out = static_cast<T *>(a.out) + q_row * a.ot + q_head * a.oh;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; k++) v[k] = none ? 0.0f : o[k];
    if (lane < kLanes && 4 * lane < c.width) store_columns<T, 4>(out, 4 * lane, c.dim, v);
    if (a.lse && lane == 0)
        a.lse[q_row * (c.heads * a.group.d) + q_head] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2E;
}

// ---- few tokens -------------------------------------------------------------
//
// A sequence with a few tokens (sampled slots) leaves the matrix instructions
// mostly idle and pays for their set-up.  Here 16 lanes serve a sequence and
// head, JV columns each, and a wavefront four of them; everything is float32.
// 16 tokens at a time: lane i looks token i up; every lane multiplies its
// columns of all 16; the products are summed over the lanes so that token i's
// sum arrives in lane i (four exchanges, halving the tokens each time); the
// weights come back from lane i by a swizzle.  12,000 roots of 10 slots, 2 heads
// of 50 float32 (23 MB): 11.8 us, half of it instructions, half the chain of
// three loads (slot, step, row); 40 us on the matrix instructions.

template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, true));
}
// Lane i's partner among 16: i ^ 8, i ^ 7, i ^ 2, i ^ 1, which together reach all.
constexpr int kXor8 = 0x128, kXor7 = 0x141, kXor2 = 0x4e, kXor1 = 0xb1;

template <int kBit, int kCtrl, int N>
__device__ __forceinline__ void scatter_sum(float (&p)[16], int i) {
#pragma unroll
    for (int k = 0; k < N; k++) {
        const float keep = i & kBit ? p[k + N] : p[k], send = i & kBit ? p[k] : p[k + N];
        p[k] = keep + dpp<kCtrl>(send);
    }
}

// Lane j of each 16.
template <int J>
__device__ __forceinline__ int from_lane(int v) {
    return __builtin_amdgcn_ds_swizzle(v, (J << 5) | 0x10);
}

constexpr float kFew = 64.0f;       // tokens at most, see few()
constexpr float kRoom = 32768.0f;   // 127 columns of 256: sums of query times bytes stay in range where scores do

template <class T, int JV>
__global__ __launch_bounds__(kBlock, (JV == 16 ? 2 : 4)) void attend_few_kernel(const AttendArgs a) {
    constexpr int kWords = JV / 4;
    const CacheView &c = a.c;
    const int i = threadIdx.x & 15;
    const uint32_t items = a.s.seqs * a.heads.d;
    const uint32_t item = (blockIdx.x * kBlock + threadIdx.x) / 16;
    const bool there = item < items;
    const uint32_t it = there ? item : items - 1;
    const uint32_t b = a.heads(it);
    const int head = static_cast<int>(it - b * a.heads.d);
    const View view = view_of_seq(a, b);
    const int64_t all = view.all, begin = view.begin, end = view.end;
    const int block = static_cast<int>(c.block_bytes());
    const uint32_t pitch = static_cast<uint32_t>(c.heads) * 2 * block;
    const int col = JV * i < c.width - JV ? JV * i : c.width - JV;
    const int8_t *data = c.data + static_cast<int64_t>(head) * 2 * block + col;
    const int pmask = c.tokens() - 1;
    const int32_t *table = a.s.table + b * a.s.table_stride;

    for (uint32_t r = 0; r < a.rows; r++) {
        const uint32_t t = a.group(r);
        const int64_t q_row = static_cast<int64_t>(b) * a.queries + t;
        const int q_head = static_cast<int>(head * a.group.d + (r - t * a.group.d));
        int64_t stop = end - (a.queries - 1 - t);
        stop = stop > all ? all : stop;
        const int n = there ? clamp_to(stop - begin, 1 << 30) : 0;
        float q[JV];
        load_columns<T, JV>(static_cast<const T *>(a.q) + q_row * a.qt + q_head * a.qh, JV * i, c.dim, q);
        bool odd = false, seen = false;             // an element that is no number; a token that is seen
#pragma unroll
        for (int k = 0; k < JV; k++) {
            q[k] *= a.scale * (kLog2E / kRoom);
            odd |= !(fabsf(q[k]) < INFINITY);
        }
        float m = -INFINITY, l = 0.0f, o[JV] = {};
        for (int j0 = 0; __any(j0 < n); j0 += 16) {
            int page = -1;
            if (j0 + i < n) page = table[(begin + j0 + i) >> c.shift];
            page = page < c.pages ? page : -1;
            const int own = page < 0 ? 0 : page;
            const float2 sc = *reinterpret_cast<const float2 *>(c.scales + (static_cast<int64_t>(own) * c.heads + head) * 2);
            const int r0 = static_cast<int>(begin + j0);
            int kw[16][kWords], vw[16][kWords];
            unrolled<16>([&](auto J) {
                constexpr int j = decltype(J)::value;
                const uint32_t at = from_lane<j>(own);
                const int8_t *k = data + static_cast<uint64_t>(at) * pitch + ((r0 + j) & pmask) * c.width;
                Columns<JV> x;
                x.load(k);
#pragma unroll
                for (int w = 0; w < kWords; w++) kw[j][w] = x.w[w];
                x.load(k + block);
#pragma unroll
                for (int w = 0; w < kWords; w++) vw[j][w] = x.w[w];
            });
            float p[16];
#pragma unroll
            for (int j = 0; j < 16; j++) {
                p[j] = 0.0f;
#pragma unroll
                for (int k = 0; k < JV; k++)
                    p[j] = __builtin_fmaf(static_cast<float>(static_cast<int8_t>(kw[j][k / 4] >> (8 * (k % 4)))), q[k], p[j]);
            }
            scatter_sum<8, kXor8, 8>(p, i);
            scatter_sum<4, kXor7, 4>(p, i);
            scatter_sum<2, kXor2, 2>(p, i);
            scatter_sum<1, kXor1, 1>(p, i);
            const float s = page < 0 ? -INFINITY : p[0] * sc.x * kRoom;
            seen |= page >= 0;
            float top = fmaxf(s, dpp<kXor8>(s));
            top = fmaxf(top, dpp<kXor7>(top));
            top = fmaxf(top, dpp<kXor2>(top));
            top = fmaxf(top, dpp<kXor1>(top));
            const float next = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - next);
            m = next;
            const float e = __builtin_amdgcn_exp2f(s - (m == -INFINITY ? 0.0f : m));
            l = l * f + e;
            const int w = __builtin_bit_cast(int, page < 0 ? 0.0f : e * (sc.y * (1.0f / kFew)));     // the sum stays below the largest value
#pragma unroll
            for (int k = 0; k < JV; k++) o[k] *= f;
            unrolled<16>([&](auto J) {
                constexpr int j = decltype(J)::value;
                const float wj = __builtin_bit_cast(float, from_lane<j>(w));
#pragma unroll
                for (int k = 0; k < JV; k++)
                    o[k] = __builtin_fmaf(static_cast<float>(static_cast<int8_t>(vw[j][k / 4] >> (8 * (k % 4)))), wj, o[k]);
            });
        }
        l += dpp<kXor8>(l);
        l += dpp<kXor7>(l);
        l += dpp<kXor2>(l);
        l += dpp<kXor1>(l);
        const bool none = group_ballot<16>(seen) == 0, bad = group_ballot<16>(odd) != 0;
        if (l == 0.0f || bad) l = __builtin_nanf("");       // every score -inf, or a query that is no number
        const float norm = kFew / l;
#pragma unroll
        for (int k = 0; k < JV; k++) o[k] = none ? 0.0f : o[k] * norm;
        if (there) {
            store_columns<T, JV>(static_cast<T *>(a.out) + q_row * a.ot + q_head * a.oh, JV * i, c.dim, o);
            if (a.lse && i == 0)
                a.lse[q_row * (c.heads * a.group.d) + q_head] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2E;
        }
    }
}

// Workgroups that fill the card a few times over; a long axis is cut until
// there are that many, into chunks of at least kMinChunk tokens, and 64 for
// each row of a tile (whose partial sums then are at most 1/16 of the bytes).
constexpr int64_t kFill = 2048;
constexpr int64_t kMinChunk = 256;

struct Plan {
    int64_t tile_rows;
    int64_t row_tiles;
    int64_t chunk;
    int64_t chunks;
    size_t part_o;          // bytes of each part of the workspace, 0 without chunks
    size_t part_ml;
};

Plan plan_of(const CacheView &c, int64_t num_seqs, int32_t pages_per_seq, int32_t q_heads, int64_t queries) {
    Plan p{};
    const int64_t rows = queries * (q_heads / c.heads);
    p.tile_rows = rows > kRows && c.width <= 128 ? 2 * kRows : kRows;
    p.row_tiles = (rows + p.tile_rows - 1) / p.tile_rows;
    const int64_t most = (static_cast<int64_t>(pages_per_seq) << c.shift) + kTile;      // begin need not be at a step's start
    const int64_t items = num_seqs * c.heads * p.row_tiles;
    int64_t chunks = items > 0 && items < kFill ? kFill / items : 1;
    const int64_t tile_rows = rows < p.tile_rows ? rows : p.tile_rows;
    const int64_t cap = most / (64 * tile_rows > kMinChunk ? 64 * tile_rows : kMinChunk);
    chunks = chunks > cap ? cap : chunks;
    const int64_t least = (most >> 30) + 1;             // positions in a chunk are 32-bit
    chunks = chunks < least ? least : chunks;
    p.chunk = (most + chunks - 1) / chunks;
    p.chunk = (p.chunk + 4 * kTile - 1) / (4 * kTile) * (4 * kTile);
    p.chunks = (most + p.chunk - 1) / p.chunk;
    if (p.chunks > 1) {
        const size_t n = static_cast<size_t>(num_seqs) * c.heads * rows * p.chunks;
        p.part_o = align_up(n * c.width * 4, 256);
        p.part_ml = align_up(n * 8, 256);
    }
    return p;
}

template <class T, int JV, int kPages>
void launch(const AttendArgs &a, int nw, hipStream_t st) {
    // whole turns of the dies, of heads or of workgroups
    const unsigned grid = a.order == kHeadsInTurn ? (a.work / a.tiles.d + 7) / 8 * 8 * a.tiles.d : (a.work + 7) / 8 * 8;
    if constexpr (JV < 16) {
        if (a.tile_rows > kRows) {
            attend_kernel<T, JV, kPages, 4, 2><<<grid, 4 * kWave, 0, st>>>(a);
            return;
        }
    }
    if (nw == 1) attend_kernel<T, JV, kPages, 1, 1><<<grid, kWave, 0, st>>>(a);
    else attend_kernel<T, JV, kPages, 4, 1><<<grid, 4 * kWave, 0, st>>>(a);
}

template <class T, int JV>
void launch(const AttendArgs &a, int nw, hipStream_t st) {
    if (a.c.tokens() >= 16) launch<T, JV, kHalves>(a, nw, st);
    else if (a.c.tokens() >= 4) launch<T, JV, kFours>(a, nw, st);
    else launch<T, JV, kTokens>(a, nw, st);
}

template <class T, int kLanes>
void launch_join(const AttendArgs &a, hipStream_t st) {
    // wavefronts of a row: enough that each has a few chunks
    if (a.chunks <= 16) attend_join_kernel<T, 1, kLanes><<<(a.all_rows + 3) / 4, kBlock, 0, st>>>(a);
    else attend_join_kernel<T, 16, kLanes><<<a.all_rows, 16 * kWave, 0, st>>>(a);
}

template <class T>
void launch(const AttendArgs &a, int nw, hipStream_t st) {
    if (a.c.width <= 32) launch<T, 2>(a, nw, st);
    else if (a.c.width <= 64) launch<T, 4>(a, nw, st);
    else if (a.c.width <= 128) launch<T, 8>(a, nw, st);
    else launch<T, 16>(a, nw, st);
    if (!a.part_o) return;
    if (a.c.width <= 64) launch_join<T, 16>(a, st);
    else if (a.c.width <= 128) launch_join<T, 32>(a, st);
    else launch_join<T, 64>(a, st);
}

// Whether the kernel for few tokens is the faster one: its work grows with
// rows times tokens, the other's with tokens above 32.  12,000 sequences, 2
// heads of 128, us here / there: 1 row of 16 tokens 23 / 51, of 32 39 / 51, of
// 64 72 / 77; 2 rows of 16 41 / 51, of 32 76 / 53; 4 rows of 8 50 / 52, of 16
// 79 / 52.
bool few(const AttendArgs &a) {
    const int64_t tokens = static_cast<int64_t>(a.s.pages_per_seq) << a.c.shift;
    return a.rows * ((tokens + 15) / 16) <= 2 || (a.rows == 1 && tokens <= static_cast<int64_t>(kFew));
}

// Wavefronts that share a sequence's tokens.  One to itself needs no join
// through LDS and leaves more of them resident, as long as there are many.  2
// heads of 50, 3 rows, us with 1 / 4: 1000 sequences and heads, 64 tokens 6.5 / 7.6,
// 128 8.1 / 9.0, 256 12.2 / 11.2; 4000 of 128 17 / 28, of 256 28 / 35, of 512
// 48 / 49; 24,000 of 256 122 / 183, of 512 227 / 264.
int wavefronts(const AttendArgs &a) {
    const int64_t tokens = static_cast<int64_t>(a.s.pages_per_seq) << a.c.shift;
    return tokens <= 64 || (tokens <= 256 && a.items.d >= 2048) ? 1 : 4;
}

template <class T>
void launch_few(const AttendArgs &a, unsigned grid, hipStream_t st) {
    if (a.c.width <= 64) attend_few_kernel<T, 4><<<grid, kBlock, 0, st>>>(a);
    else if (a.c.width <= 128) attend_few_kernel<T, 8><<<grid, kBlock, 0, st>>>(a);
    else attend_few_kernel<T, 16><<<grid, kBlock, 0, st>>>(a);
}

// The part of a call that is n sequences from b on.
AttendArgs slice(AttendArgs a, int64_t b, int64_t n, size_t elem) {
    const int64_t row = b * a.queries, items = n * a.c.heads;
    a.s.table += b * a.s.table_stride;
    if (a.s.start) a.s.start += b;
    if (a.end) a.end += b;
    a.s.seqs = static_cast<int32_t>(n);
    a.q = static_cast<const char *>(a.q) + row * a.qt * static_cast<int64_t>(elem);
    a.out = static_cast<char *>(a.out) + row * a.ot * static_cast<int64_t>(elem);
    if (a.lse) a.lse += row * a.c.heads * a.group.d;
    a.items = Div(static_cast<uint32_t>(items));
    a.work = static_cast<uint32_t>(items * a.tiles.d * a.chunks);
    a.all_rows = static_cast<uint32_t>(items * a.rows);
    const int64_t units = items * a.chunks;
    a.order = a.tiles.d == 1 ? kInTurn : units >= 32 || units % 8 == 0 ? kHeadsInTurn : kStretches;
    return a;
}

template <class T>
void launch(const AttendArgs &a, hipStream_t st) {
    if (few(a)) launch_few<T>(a, static_cast<unsigned>((a.items.d + 15) / 16), st);
    else launch<T>(a, wavefronts(a), st);
}

// Rows without anything to see: zeros.
template <class T>
__global__ __launch_bounds__(kBlock) void attend_none_kernel(const AttendArgs a) {
    const int heads = a.c.heads * a.group.d;
    const int64_t n = static_cast<int64_t>(a.s.seqs) * a.queries * heads * a.c.dim;
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
    AttendArgs a{};
    a.c = view_of(*cache);
    a.s = view_of(*seqs, rows);
    a.end = end;
    a.q = q->ptr;
    a.out = out->ptr;
    a.lse = lse;
    a.qt = q->token_stride;
    a.qh = q->head_stride;
    a.ot = out->token_stride;
    a.oh = out->head_stride;
    a.queries = static_cast<uint32_t>(queries);
    a.scale = scale;
    const uint32_t group = q_heads / cache->heads;
    a.group = Div(group);
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
    a.rows = static_cast<uint32_t>(queries * group);
    a.row_of = Div(a.rows);
    a.chunk = p.chunk;
    a.tile_rows = static_cast<uint32_t>(p.tile_rows);
    a.tiles = Div(static_cast<uint32_t>(p.row_tiles));
    a.chunks = static_cast<uint32_t>(p.chunks);
    a.heads = Div(a.c.heads);
    if (p.part_o) {
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part_o);
    }
    // A launch has fewer than 2^32 threads: as many sequences at a time as keep
    // to that.  Their launches follow each other, so they share the workspace.
    int64_t most = ((int64_t(1) << 24) - 1 - 8 * p.row_tiles) / (a.c.heads * p.row_tiles * p.chunks);   // of 256 threads
    const int64_t joins = ((int64_t(1) << 22) - 1) / (static_cast<int64_t>(a.c.heads) * a.rows);        // of 1024
    if (p.part_o && most > joins) most = joins;
    if (most < 1) return TGL_EINVAL;
    for (int64_t b = 0; b < seqs->num_seqs; b += most) {
        const AttendArgs part = slice(a, b, seqs->num_seqs - b < most ? seqs->num_seqs - b : most, elem_size(dtype));
        if (dtype == TGL_OUT_F32) launch<float>(part, st);
        else launch<bf16_t>(part, st);
        if (launch_status() != TGL_OK) return TGL_EDEVICE;
    }
    return TGL_OK;
}

}  // extern "C"
