// tgl_groups.hip -- rows sorted by their type: a counting sort whose result
// does not depend on the order of any two wavefronts.
//
//   bin(i) = type of row i, or num_types for rows of no type
//   order  = rows by (bin, row);  offsets[g] = number of rows of a bin below g
//
// A wavefront owns consecutive rows and walks them 64 at a time: the lanes
// whose bins are equal find each other with one ballot for each bit of a bin,
// so a row's rank among its wavefront's rows of that bin is the bin's count so far
// plus the set bits below the lane.
#include "tgl_internal.hpp"

namespace tgl {
namespace {

constexpr int kWaves = 16;                  // of a workgroup here
constexpr int kThreads = kWaves * kWave;
constexpr int kAhead = 8;                   // rows a lane holds
constexpr int kFew = 2 * kAhead * kThreads; // rows that one workgroup sorts
constexpr int kBins = TGL_MAX_TYPES + 1;

struct GroupArgs {
    const void *types;
    const int32_t *ids;
    int64_t num_ids;
    int64_t n;
    int32_t *order;
    int64_t *offsets;
    uint32_t *counts;       // [bins][pitch]: rows of a bin in a wavefront's chunk, then in all chunks before it
    uint32_t *totals;       // [bins]
    uint16_t *kept;         // bins that were looked up, or null
    int32_t num_types;
    int32_t bits;           // of a bin
    int32_t chunk;          // rows of a wavefront
    int32_t chunks;
    int32_t pitch;          // chunks, rounded up to 8
};

template <class K>
__device__ __forceinline__ uint32_t bin_of(const GroupArgs &a, int64_t row) {
    int64_t t;
    if (a.ids) {
        const int32_t id = __builtin_nontemporal_load(a.ids + row);       // read once: the nodes' types stay in the caches
        t = id >= 0 && id < a.num_ids ? static_cast<const K *>(a.types)[id] : -1;
    } else {
        t = static_cast<const K *>(a.types)[row];
    }
    return t >= 0 && t < a.num_types ? static_cast<uint32_t>(t) : a.num_types;
}

// The lanes of `among` whose bin is the calling lane's.
__device__ __forceinline__ uint64_t same_bin(uint32_t bin, int bits, uint64_t among) {
    for (int b = 0; b < bits; b++) {
        const uint64_t set = __ballot((bin >> b) & 1);
        among &= (bin >> b) & 1 ? set : ~set;
    }
    return among;
}

// Adds one row a lane to the wavefront's counts; a row's own count before it.
__device__ __forceinline__ uint32_t count_row(uint32_t *count, uint32_t bin, int bits, bool there) {
    const uint64_t same = same_bin(bin, bits, __ballot(there));
    const int first = __builtin_ctzll(same | (1ull << 63));
    uint32_t before = 0;
    if (there && lane_id() == first) before = atomicAdd(&count[bin], static_cast<uint32_t>(__popcll(same)));
    return __shfl(before, first, kWave) + rank_below(same);
}

// Exclusive sum over the workgroup's threads.
__device__ __forceinline__ uint32_t before_thread(uint32_t v, uint32_t *parts) {
    const uint32_t inc = wave_inclusive_sum(v);
    if (lane_id() == kWave - 1) parts[threadIdx.x / kWave] = inc;
    __syncthreads();
    uint32_t sum = inc - v;
    for (int w = 0; w < static_cast<int>(threadIdx.x / kWave); w++) sum += parts[w];
    __syncthreads();
    return sum;
}

// Up to 16,384 rows in one workgroup, a launch in all: a batch of 1800 roots
// of 3 types waits for memory twice and for LDS a few times.
template <class K, int N>
__global__ __launch_bounds__(kThreads) void group_few_kernel(const GroupArgs a) {
    __shared__ uint32_t count[kWaves][kBins];
    __shared__ uint32_t begin[kBins];
    __shared__ uint32_t parts[kWaves];
    const int wave = threadIdx.x / kWave;
    const int bins = a.num_types + 1;
    const int n = static_cast<int>(a.n);
    for (int b = lane_id(); b < bins; b += kWave) count[wave][b] = 0;
    const int first = wave * N * kWave + lane_id();
    uint32_t bin[N], rank[N];
#pragma unroll
    for (int i = 0; i < N; i++) bin[i] = first + i * kWave < n ? bin_of<K>(a, first + i * kWave) : 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) rank[i] = count_row(count[wave], bin[i], a.bits, first + i * kWave < n);
    __syncthreads();
    // a bin's rows in the wavefronts before, and in all
    const int b = threadIdx.x;
    uint32_t sum = 0;
    if (b < a.num_types) {
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            const uint32_t c = count[w][b];
            count[w][b] = sum;
            sum += c;
        }
    }
    const uint32_t at = before_thread(sum, parts);
    if (b < a.num_types) {
        begin[b] = at;
        a.offsets[b] = at;
    }
    if (b == kThreads - 1) {                // the last bin, of rows without a type
        begin[a.num_types] = at + sum;
        a.offsets[a.num_types] = at + sum;
        uint32_t none = 0;
        for (int w = 0; w < kWaves; w++) {
            const uint32_t c = count[w][a.num_types];
            count[w][a.num_types] = none;
            none += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++)
        if (first + i * kWave < n) a.order[begin[bin[i]] + count[wave][bin[i]] + rank[i]] = first + i * kWave;
}

// Rows of every bin in every wavefront's chunk.  What ids look up is kept, so
// that the types of random nodes are fetched once.
template <class K>
__global__ __launch_bounds__(kThreads) void group_count_kernel(const GroupArgs a) {
    __shared__ uint32_t count[kWaves][kBins];
    const int wave = threadIdx.x / kWave;
    const int64_t chunk = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    const int bins = a.num_types + 1;
    for (int b = lane_id(); b < bins; b += kWave) count[wave][b] = 0;
    __syncthreads();
    if (chunk >= a.chunks) return;
    const int64_t end = (chunk + 1) * a.chunk < a.n ? (chunk + 1) * a.chunk : a.n;
    for (int64_t row = chunk * a.chunk + lane_id(); row < end + lane_id(); row += kAhead * kWave) {
        uint32_t bin[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) bin[i] = row + i * kWave < end ? bin_of<K>(a, row + i * kWave) : 0;
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const bool there = row + i * kWave < end;
            if (a.kept && there) a.kept[row + i * kWave] = static_cast<uint16_t>(bin[i]);
            const uint64_t same = same_bin(bin[i], a.bits, __ballot(there));
            if (there && rank_below(same) == 0) atomicAdd(&count[wave][bin[i]], static_cast<uint32_t>(__popcll(same)));
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int b = lane_id(); b < bins; b += kWave) a.counts[static_cast<int64_t>(b) * a.pitch + chunk] = count[wave][b];
}

// A workgroup per bin: its rows in all chunks before each, and in all.  A thread has 8
// chunks, of the 8192 at most.
__global__ __launch_bounds__(kThreads) void group_scan_kernel(const GroupArgs a) {
    using four_t = uint32_t __attribute__((ext_vector_type(4)));
    __shared__ uint32_t parts[kWaves];
    const int first = threadIdx.x * 8;
    four_t *count = reinterpret_cast<four_t *>(a.counts + static_cast<int64_t>(blockIdx.x) * a.pitch + first);
    four_t v[2] = {};
    if (first < a.pitch) {
        v[0] = count[0];
        v[1] = count[1];
    }
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (first + i >= a.chunks) v[i / 4][i % 4] = 0;             // what lies behind the chunks
        sum += v[i / 4][i % 4];
    }
    uint32_t at = before_thread(sum, parts);
    if (threadIdx.x == kThreads - 1) a.totals[blockIdx.x] = at + sum;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t own = v[i / 4][i % 4];
        v[i / 4][i % 4] = at;
        at += own;
    }
    if (first < a.pitch) {
        count[0] = v[0];
        count[1] = v[1];
    }
}

// Every row to its place.
template <class K>
__global__ __launch_bounds__(kThreads) void group_place_kernel(const GroupArgs a) {
    __shared__ uint32_t count[kWaves][kBins];
    __shared__ uint32_t begin[kBins];
    __shared__ uint32_t parts[kWaves];
    const int wave = threadIdx.x / kWave;
    const int64_t chunk = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    const int bins = a.num_types + 1;
    const int t = threadIdx.x;
    const uint32_t total = t < a.num_types ? a.totals[t] : 0;
    const uint32_t at = before_thread(total, parts);
    if (t < a.num_types) begin[t] = at;
    if (t == kThreads - 1) begin[a.num_types] = at + total;
    __syncthreads();
    if (blockIdx.x == 0)
        for (int b = t; b < bins; b += kThreads) a.offsets[b] = begin[b];
    if (chunk >= a.chunks) return;
    for (int b = lane_id(); b < bins; b += kWave)
        count[wave][b] = begin[b] + a.counts[static_cast<int64_t>(b) * a.pitch + chunk];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int64_t end = (chunk + 1) * a.chunk < a.n ? (chunk + 1) * a.chunk : a.n;
    for (int64_t row = chunk * a.chunk + lane_id(); row < end + lane_id(); row += kAhead * kWave) {
        uint32_t bin[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            bin[i] = 0;
            if (row + i * kWave < end) bin[i] = a.kept ? a.kept[row + i * kWave] : bin_of<K>(a, row + i * kWave);
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const bool there = row + i * kWave < end;
            const uint32_t place = count_row(count[wave], bin[i], a.bits, there);
            if (there) a.order[place] = static_cast<int32_t>(row + i * kWave);
        }
    }
}

// Rows of a wavefront's chunk: so many that there are 8192 chunks at most, 2048 as long as a
// chunk has 128 rows (counting 120,000 slots 7 us, in chunks of 512 16), and fewer counts than a
// quarter of the rows.
int64_t chunk_rows(int64_t n, int32_t num_types) {
    int64_t rows = (n + 8191) / 8192;
    const int64_t spread = n / 2048 < 128 ? 128 : n / 2048 < 512 ? n / 2048 : 512;
    if (rows < spread) rows = spread;
    if (rows < 4 * num_types) rows = 4 * num_types;
    return (rows + kWave - 1) / kWave * kWave;
}

size_t carve(GroupArgs &a, void *base) {
    Carver c(base);
    a.counts = c.take<uint32_t>(static_cast<size_t>(a.pitch) * (a.num_types + 1));
    a.totals = c.take<uint32_t>(kBins);
    a.kept = c.take<uint16_t>(static_cast<size_t>(a.n));
    return c.size();
}

bool split(GroupArgs &a) {
    if (a.n <= kFew) return false;
    a.chunk = static_cast<int32_t>(chunk_rows(a.n, a.num_types));
    a.chunks = static_cast<int32_t>((a.n + a.chunk - 1) / a.chunk);
    a.pitch = (a.chunks + 7) & ~7;
    return true;
}

template <class K>
tgl_status launch_group(const GroupArgs &a, hipStream_t st) {
    if (a.n <= 2 * kThreads) {
        group_few_kernel<K, 2><<<1, kThreads, 0, st>>>(a);
        return launch_status();
    }
    if (a.n <= kFew) {
        group_few_kernel<K, 2 * kAhead><<<1, kThreads, 0, st>>>(a);
        return launch_status();
    }
    const unsigned blocks = static_cast<unsigned>((a.chunks + kWaves - 1) / kWaves);
    group_count_kernel<K><<<blocks, kThreads, 0, st>>>(a);
    if (launch_status() != TGL_OK) return TGL_EDEVICE;
    group_scan_kernel<<<static_cast<unsigned>(a.num_types + 1), kThreads, 0, st>>>(a);
    if (launch_status() != TGL_OK) return TGL_EDEVICE;
    group_place_kernel<K><<<blocks, kThreads, 0, st>>>(a);
    return launch_status();
}

bool valid_counts(int64_t n, int32_t num_types) {
    return n >= 0 && n < (int64_t(1) << 31) && num_types >= 1 && num_types <= TGL_MAX_TYPES;
}

inline bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace tgl

using namespace tgl;

extern "C" {

size_t tgl_group_rows_workspace(int64_t n, int32_t num_types) {
    if (!valid_counts(n, num_types)) return 0;
    GroupArgs a{};
    a.n = n;
    a.num_types = num_types;
    return split(a) ? carve(a, nullptr) : 0;
}

tgl_status tgl_group_rows(const void *types, int32_t types64, int64_t num_ids, const int32_t *ids, int64_t n,
                          int32_t num_types, int32_t *order, int64_t *offsets, void *workspace,
                          size_t workspace_bytes, void *stream) {
    if (!valid_counts(n, num_types) || (types64 != 0 && types64 != 1)) return TGL_EINVAL;
    if (ids && num_ids < 0) return TGL_EINVAL;
    if (!aligned_to(types, types64 ? 8 : 4) || !aligned_to(ids, 4) || !aligned_to(order, 4) || !aligned_to(offsets, 8))
        return TGL_EINVAL;
    if (!offsets || (n > 0 && !order)) return TGL_EINVAL;
    if ((ids ? num_ids : n) > 0 && !types) return TGL_EINVAL;
    GroupArgs a{};
    a.types = types;
    a.ids = ids;
    a.num_ids = num_ids;
    a.n = n;
    a.order = order;
    a.offsets = offsets;
    a.num_types = num_types;
    a.bits = 32 - __builtin_clz(static_cast<uint32_t>(num_types));
    if (split(a)) {
        if (!workspace || workspace_bytes < carve(a, nullptr)) return TGL_ENOSPACE;
        if (!aligned_to(workspace, 256)) return TGL_EINVAL;
        carve(a, workspace);
        if (!ids) a.kept = nullptr;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    return types64 ? launch_group<int64_t>(a, st) : launch_group<int32_t>(a, st);
}

}  // extern "C"
