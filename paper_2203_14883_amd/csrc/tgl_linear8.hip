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
    Div tiles_n;            // small products: tiles of 16 columns
    Div band;               // large ones: tiles of a band of band_rows tiles of rows
    uint32_t band_rows, tiles_m, work;
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

// An int32 sum, which of 2^17 products of -128 with itself is 2^31: no other sum
// has those bits, since the least is -128 * 127 * 2^17.
__device__ __forceinline__ float sum_of(int v) { return v == INT32_MIN ? 0x1p31f : static_cast<float>(v); }

// Scales, bias, the one rounding: N outputs of a row from column j on.
template <class T, int N>
__device__ __forceinline__ void finish(const LinearArgs &a, int64_t row, int j, const int (&sum)[N], const float (&ws)[N], const float (&bias)[N]) {
    const float xs = a.xs[row];
    float y[N];
#pragma unroll
    for (int i = 0; i < N; i++) {
        y[i] = sum_of(sum[i]) * xs * ws[i];
        if (a.bias) y[i] += bias[i];
    }
    store_columns<T, N>(static_cast<T *>(a.out) + row * a.ostride, j, a.n, y);
}

// ---- small products: operands straight from memory --------------------------

// A workgroup per 16 MT rows and 16 columns, whose wavefronts take 64 of k in
// turn and add up through LDS: a row of w is read once for 16 MT rows of x.
// Bound by latency where w is small (1 x 2304 x 768: 3.4 us) and by w's bytes
// where it is not (1 x 4096 x 4096: 4.8 us, 3.5 TB/s).
template <class T, int NW, int MT>
__global__ __launch_bounds__(NW * kWave) void linear_small_kernel(const LinearArgs a) {
    __shared__ i32x4 sums[NW > 1 ? NW : 1][MT][kWave];
    const int lane = lane_id();
    const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t tm = a.tiles_n(blockIdx.x), tn = blockIdx.x - tm * a.tiles_n.d;
    const int64_t m0 = static_cast<int64_t>(tm) * (16 * MT);
    const int n0 = tn * 16;
    const int nr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const int8_t *w = a.w + nr * a.wstride;
    const int8_t *x[MT];
    i32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int64_t mr = m0 + 16 * i + (lane & 15);
        x[i] = a.x + (mr < a.m ? mr : a.m - 1) * a.xstride;
        acc[i] = i32x4{0, 0, 0, 0};
    }
    // whole steps of 64 with nothing to check, then the rest of k
    const int whole = a.k & ~63;
    constexpr int kUnroll = MT == 1 ? 4 : 2;
    int k = wave * 64;
    for (; k + (kUnroll - 1) * NW * 64 < whole; k += kUnroll * NW * 64) {
        i32x4 wv[kUnroll], xv[kUnroll][MT];
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const int c = k + u * NW * 64 + 16 * (lane >> 4);
            wv[u] = *reinterpret_cast<const i32x4 *>(w + c);
#pragma unroll
            for (int i = 0; i < MT; i++) xv[u][i] = *reinterpret_cast<const i32x4 *>(x[i] + c);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; u++)
#pragma unroll
            for (int i = 0; i < MT; i++) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u], xv[u][i], acc[i], 0, 0, 0);
    }
    for (; k < a.k; k += NW * 64) {
        const int c = k + 16 * (lane >> 4);
        const i32x4 wv = load_piece(w, c, a.k);
#pragma unroll
        for (int i = 0; i < MT; i++)
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, mask_piece(load_piece(x[i], c, a.k), c, a.k), acc[i], 0, 0, 0);
    }
    const int j = n0 + 4 * (lane >> 4);
    float ws[4], bias[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int col = j + i < a.n ? j + i : a.n - 1;
        ws[i] = a.ws[col];
        bias[i] = a.bias ? a.bias[col] : 0.0f;
    }
    auto put = [&](int i, const i32x4 &v) {
        const int64_t row = m0 + 16 * i + (lane & 15);
        if (row >= a.m || j >= a.n) return;
        const int sum[4] = {v[0], v[1], v[2], v[3]};
        finish<T, 4>(a, row, j, sum, ws, bias);
    };
    if constexpr (NW == 1) {
#pragma unroll
        for (int i = 0; i < MT; i++) put(i, acc[i]);
    } else {
#pragma unroll
        for (int i = 0; i < MT; i++) sums[wave][i][lane] = acc[i];
        __syncthreads();
        for (int i = wave; i < MT; i += NW) {       // a wavefront finishes a row tile
            i32x4 v = sums[0][i][lane];
#pragma unroll
            for (int y = 1; y < NW; y++) v += sums[y][i][lane];
            put(i, v);
        }
    }
}

// ---- large products: tiles through LDS --------------------------------------
//
// A workgroup owns BM x BN outputs and walks k in steps of 128: a step's
// BM + BN rows of 128 bytes go straight from memory to one of S LDS buffers,
// S - 1 steps ahead of the one that is multiplied.  A wavefront owns 64 columns and MT x 16 rows;
// the weights are the first operand, so that a lane ends up with columns of
// one row, and its four tiles' rows of w are picked so that these are 16
// consecutive ones: 4 of each (lane / 16) * 16 + 4 tile + 0..3.
//
// A 16-byte piece p of row r lies at piece p ^ swizzle(r) of the row's 128
// bytes, so that the 16 lanes that read one piece of 16 rows touch all banks.
// Whole pieces only: past them LDS holds 0, from loads beyond the buffer's end,
// and a piece that k ends in is multiplied once, after the steps, from memory.

// Bound by the matrix units and their feeding: 16384 x 4096 x 4096 in 252 to 272
// us by the card's clocks, 2.0 to 2.2 POP/s, the units at work 47% of the time;
// 8192^3 in 413 us, 2.7 POP/s.  One row of 65,536 columns (128 x 128 tiles, of
// 268 MB of weights) 41 us, 6.5 TB/s.  The steps overlap: loads, 6 reads of LDS for every 8
// products, and the products of two wavefronts a SIMD.

constexpr int kStepK = 128;

__device__ __forceinline__ int swizzle_x(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int swizzle_w(int r) { return ((r >> 1) & 1) | (((r >> 4) & 3) << 1); }

using lds_t = __attribute__((address_space(3))) void;

template <class T, int BM, int BN, int MT, int S>
__global__ __launch_bounds__(BM / (16 * MT) * (BN / 64) * kWave, 2) void linear_tile_kernel(const LinearArgs a) {
    constexpr int kWaves = BM / (16 * MT) * (BN / 64);
    constexpr int kFetchW = BN / 8 / kWaves, kFetch = kFetchW + BM / 8 / kWaves;    // fetches of 8 rows of w, of all
    static_assert(BN % (8 * kWaves) == 0 && BM % (8 * kWaves) == 0, "the wavefronts fetch as much each");
    // one object each: so the compiler sees that a step's reads do not wait for the others' loads
    __shared__ __attribute__((aligned(1024))) int8_t buf0[(BM + BN) * kStepK];
    __shared__ __attribute__((aligned(1024))) int8_t buf1[(BM + BN) * kStepK];
    __shared__ __attribute__((aligned(1024))) int8_t buf2[S > 2 ? (BM + BN) * kStepK : 16];
    __shared__ __attribute__((aligned(1024))) int8_t buf3[S > 3 ? (BM + BN) * kStepK : 16];
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int g = lane >> 4, i16 = lane & 15;
    // the 8 dies take workgroups in turn: each gets a contiguous stretch of
    // tiles, walked in bands of band_rows tiles of rows
    const uint32_t per = (a.work + 7) / 8;
    const uint32_t id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || id >= a.work) return;
    const uint32_t band = a.band(id);                       // tiles_n * band_rows tiles
    const uint32_t in_band = id - band * a.band.d;
    const uint32_t rows_left = a.tiles_m - band * a.band_rows;
    const uint32_t height = rows_left < a.band_rows ? rows_left : a.band_rows;
    const uint32_t tn = in_band / height, tm = band * a.band_rows + (in_band - tn * height);
    const int64_t m0 = static_cast<int64_t>(tm) * BM;
    const int n0 = tn * BN;

    // ---- what the wavefront fetches ----
    const int whole = a.k & ~15;                            // what goes through LDS
    const int last_w = (a.n - n0 < BN ? a.n - n0 : BN) - 1;             // the tile's last rows
    const int last_x = static_cast<int>(a.m - m0 < BM ? a.m - m0 : BM) - 1;
    const auto rsrc_w = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.w + static_cast<int64_t>(n0) * a.wstride), 0,
                                                          last_w * static_cast<uint32_t>(a.wstride) + whole, 0x00027000);
    const auto rsrc_x = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.x + m0 * a.xstride), 0,
                                                          last_x * static_cast<uint32_t>(a.xstride) + whole, 0x00027000);
    uint32_t at[kFetch];
    uint32_t piece[kFetch];
#pragma unroll
    for (int f = 0; f < kFetch; f++) {
        const bool of_w = f < kFetchW;
        const int r = (of_w ? wave * kFetchW + f : wave * (kFetch - kFetchW) + f - kFetchW) * 8 + (lane >> 3);
        const int last = of_w ? last_w : last_x;
        piece[f] = ((lane & 7) ^ (of_w ? swizzle_w(r) : swizzle_x(r))) * 16;
        at[f] = (r < last ? r : last) * static_cast<uint32_t>(of_w ? a.wstride : a.xstride) + piece[f];
    }
    const int steps = (whole + kStepK - 1) / kStepK;
    auto fetch = [&](int8_t *buf, int step) {
        const uint32_t k = step * kStepK;
#pragma unroll
        for (int f = 0; f < kFetch; f++) {
            // beyond the row: past the buffer's end, which reads as 0
            const uint32_t off = k + piece[f] < static_cast<uint32_t>(whole) ? at[f] + k : 0x7ffffff0u;
            if (f < kFetchW)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_w, (lds_t *)(buf + (wave * kFetchW + f) * 8 * kStepK), 16, off, 0, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rsrc_x, (lds_t *)(buf + (BN + (wave * (kFetch - kFetchW) + f - kFetchW) * 8) * kStepK), 16, off, 0, 0, 0);
        }
    };

    // ---- what it multiplies ----
    const int wm = wave / (BN / 64), wn = wave % (BN / 64);
    i32x4 acc[MT][4];
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = i32x4{0, 0, 0, 0};
    int w_at[4], x_at[MT];
#pragma unroll
    for (int j = 0; j < 4; j++) w_at[j] = wn * 64 + (i16 >> 2) * 16 + 4 * j + (i16 & 3);
#pragma unroll
    for (int i = 0; i < MT; i++) x_at[i] = wm * 16 * MT + 16 * i + i16;
    auto multiply = [&](const int8_t *buf) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int p = 4 * h + g;
            i32x4 wv[4], xv[MT];
#pragma unroll
            for (int j = 0; j < 4; j++)
                wv[j] = *reinterpret_cast<const i32x4 *>(buf + w_at[j] * kStepK + ((p ^ swizzle_w(w_at[j])) * 16));
#pragma unroll
            for (int i = 0; i < MT; i++)
                xv[i] = *reinterpret_cast<const i32x4 *>(buf + (BN + x_at[i]) * kStepK + ((p ^ swizzle_x(x_at[i])) * 16));
#pragma unroll
            for (int i = 0; i < MT; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j], xv[i], acc[i][j], 0, 0, 0);
        }
    };
    // Loads to LDS count as loads from memory: each wavefront waits for its own
    // of a step, leaving the S - 2 later steps' on their way, then for the
    // others.  Steps beyond k are fetched too (nothing but zeros, from no
    // memory), so that there are always as many.
    constexpr int kLeft = (S - 2) * kFetch;
    static_assert(kLeft < 64, "the counter has six bits");
    auto meet = [] {
        // __syncthreads and fences would wait for every load: the wait and the
        // barrier by themselves, with nothing moved across them
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (kLeft & 15) | ((kLeft >> 4) << 14));      // vmcnt(kLeft), lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto buffer = [&](auto I) -> int8_t * {
        constexpr int i = decltype(I)::value % S;
        if constexpr (i == 0) return buf0;
        else if constexpr (i == 1) return buf1;
        else if constexpr (i == 2) return buf2;
        else return buf3;
    };
    unrolled<S - 1>([&](auto I) { fetch(buffer(I), decltype(I)::value); });
    for (int step = 0; step < steps; step += S) {
        unrolled<S>([&](auto I) {
            constexpr int i = decltype(I)::value;
            if (step + i < steps) {
                meet();                                     // this step's buffer is there, the one before free
                fetch(buffer(Const<i + S - 1>()), step + i + S - 1);
                multiply(buffer(I));
            }
        });
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                     // nothing goes to LDS once it is another workgroup's

    if (a.k % 16 != 0) {                                    // the piece that k ends in, straight from memory
        i32x4 wv[4], xv[MT];
        const int c = g == 0 ? whole : a.k;                 // the other lanes' pieces lie past k: zeros
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int r = w_at[j] < last_w ? w_at[j] : last_w;
            wv[j] = load_piece(a.w + (n0 + r) * a.wstride, c, a.k);
        }
#pragma unroll
        for (int i = 0; i < MT; i++) {
            const int r = x_at[i] < last_x ? x_at[i] : last_x;
            xv[i] = mask_piece(load_piece(a.x + (m0 + r) * a.xstride, c, a.k), c, a.k);
        }
#pragma unroll
        for (int i = 0; i < MT; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j], xv[i], acc[i][j], 0, 0, 0);
    }

    const int j0 = n0 + wn * 64 + 16 * g;
    if (j0 >= a.n) return;
    float ws[16], bias[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int col = j0 + i < a.n ? j0 + i : a.n - 1;
        ws[i] = a.ws[col];
        bias[i] = a.bias ? a.bias[col] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int64_t row = m0 + x_at[i];
        if (row < a.m) {
            int sum[16];
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) sum[4 * j + e] = acc[i][j][e];
            finish<T, 16>(a, row, j0, sum, ws, bias);
        }
    }
}

template <class T, int BM, int BN, int MT, int S>
void launch_tiles(LinearArgs a, hipStream_t st) {
    constexpr int kThreads = BM / (16 * MT) * (BN / 64) * kWave;
    const uint32_t tiles_n = (a.n + BN - 1) / BN;
    a.tiles_m = static_cast<uint32_t>((a.m + BM - 1) / BM);
    a.work = a.tiles_m * tiles_n;
    a.band_rows = 8;
    a.band = Div(tiles_n * a.band_rows);
    const unsigned grid = (a.work + 7) / 8 * 8;
    linear_tile_kernel<T, BM, BN, MT, S><<<grid, kThreads, 0, st>>>(a);
}

template <class T, int MT>
void launch_small(LinearArgs a, hipStream_t st) {
    a.tiles_n = Div((a.n + 15) / 16);
    const unsigned grid = static_cast<unsigned>((a.m + 16 * MT - 1) / (16 * MT) * a.tiles_n.d);
    // wavefronts that share a tile's k, while tiles alone do not fill the card
    if (a.k <= 64) linear_small_kernel<T, 1, MT><<<grid, kWave, 0, st>>>(a);
    else if (grid >= 1024 || a.k <= 512) linear_small_kernel<T, 4, MT><<<grid, 4 * kWave, 0, st>>>(a);
    else linear_small_kernel<T, 8, MT><<<grid, 8 * kWave, 0, st>>>(a);
}

template <class T>
void launch(const LinearArgs &a, hipStream_t st) {
    auto tiles = [&](int b) { return (a.m + b - 1) / b * ((a.n + b - 1) / b); };
    // The largest tiles that still give most of the 256 compute units one
    // (fewer loads a product), two workgroups a unit for those of 128; tiles of
    // 64, three steps ahead, for the middle; straight from memory where there
    // would be few of those.  Times in us with tiles of 256 / 128 / 64 / none:
    // 16384 x 4096 x 512 63 / 69 / 119 / 295, 12000 x 1024 x 768 21 / 19 / 30 /
    // 87, 2048 x 2048 x 2048 32 / 15 / 18 / 74, 512 x 4096 x 4096 50 / 26 / 16 /
    // 74, 64 x 4096 x 4096 41 / 18 / 10 / 11, 48 x 1000 x 2000 22 / 10 / 7 / 4.
    const bool fits = tiles(256) * 4 * 10 <= tiles(128) * 11;          // at most a tenth more of the edges
    if (tiles(256) >= 192 && fits) launch_tiles<T, 256, 256, 8, 2>(a, st);
    else if (tiles(128) >= 256) launch_tiles<T, 128, 128, 2, 2>(a, st);
    else if (a.m > 32 && tiles(64) >= 64) launch_tiles<T, 64, 64, 1, 4>(a, st);
    else if (a.m <= 16) launch_small<T, 1>(a, st);
    else launch_small<T, 2>(a, st);
}

// A launch has fewer than 2^32 threads: as many rows at a time as keep to that
// with tiles of 64 and 256 threads, or of 128 and 512.
template <class T>
tgl_status launch_parts(LinearArgs a, hipStream_t st) {
    const int64_t most = (int64_t(1) << 25) / ((a.n + 15) / 16) / 16 * 256, all = a.m;
    for (int64_t row = 0; row < all; row += most) {
        a.m = all - row < most ? all - row : most;
        launch<T>(a, st);
        if (launch_status() != TGL_OK) return TGL_EDEVICE;
        a.x += most * a.xstride;
        a.xs += most;
        a.out = static_cast<T *>(a.out) + most * a.ostride;
    }
    return TGL_OK;
}

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

tgl_status tgl_linear_i8(const int8_t *x, int64_t x_stride, const float *x_scale, int64_t m, const int8_t *w,
                         int64_t w_stride, const float *w_scale, const float *bias, int32_t n, int32_t k,
                         void *out, int64_t out_stride, int32_t out_type, void *stream) {
    if (m < 0 || n < 1 || n > TGL_MAX_LINEAR_OUT || k < 1 || k > TGL_MAX_LINEAR_K || !is_elem_type(out_type))
        return TGL_EINVAL;
    if (!aligned(x, 16) || !aligned(w, 16) || x_stride % 16 != 0 || w_stride % 16 != 0 || x_stride < 0 || w_stride < 0 ||
        x_stride >= (1 << 22) || w_stride >= (1 << 22))
        return TGL_EINVAL;
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(out, elem_size(out_type)))
        return TGL_EINVAL;
    if (m > 0 && (!x || !x_scale || !w || !w_scale || !out || out_stride < n)) return TGL_EINVAL;
    if (m == 0) return TGL_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    LinearArgs a{};
    a.x = x;
    a.w = w;
    a.xs = x_scale;
    a.ws = w_scale;
    a.bias = bias;
    a.out = out;
    a.xstride = x_stride;
    a.wstride = w_stride;
    a.ostride = out_stride;
    a.m = m;
    a.n = n;
    a.k = k;
    return out_type == TGL_OUT_F32 ? launch_parts<float>(a, st) : launch_parts<bf16_t>(a, st);
}

}  // extern "C"
