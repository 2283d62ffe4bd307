// Gradient of a lookup with respect to the table's rows:
//   grad[r, :] = scale * sum over the ids i that name row r of grad_out[bag(i), :].
//
// The ids are sorted by row, stably, with the row of grad_out that each stands
// for; equal ids then lie side by side, and each run of them is summed in fp32
// in the order of the ids.  No value is added to by an atomic, so the result is
// the same from call to call.
//
// Launches cost a small call more than its work, so there are three sequences:
//   few ids and values: one kernel, which finds equal ids by comparing;
//   up to 8,192 ids: every id's place by comparing it with all others, sums, joins;
//   more: radix passes of at most 10 bits over tiles of 4,096 ids (count the digits
//   of each tile, then place each id behind the smaller digits, the same digit in
//   earlier tiles, earlier waves and earlier lanes), sums, joins.
// Sums: the sorted ids are cut into chunks of equal length whatever the runs, so
// a token that a tenth of a batch repeats takes no longer than others (4 million
// ids of 16 fp32 columns: 480 us without one, 466 with a tenth, 471 with half, 553
// where all are one; 1 million of 64 columns: 169, 168, 209, 268: the run's many
// partial sums are joined by one block per 1,024 columns).  A group
// of lanes sums a chunk's runs for one slice of the columns; a run that lies in
// one chunk goes straight to its row, the ends of the others to fp32 partial
// sums that one more kernel adds up.  Rows that no id names are cleared by more
// blocks of the kernel that sums: they look their rows up in the sorted ids.
#include <type_traits>

#include "embedding.h"
#include "recmg_device.h"
#include "values.h"

namespace recmg {

namespace {

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64, kKeysPerThread = kSortTile / kSortBlock;
constexpr int kWaveKeys = kSortTile / kSortWaves;  // consecutive ids of one wave
constexpr int kBins = 1 << kMaxDigit;
constexpr int kSumBlock = 256, kDirectBlock = 512;
constexpr int kMaxZeroRows = 512;  // rows of a clearing block
// Sorted ids per chunk: few where comparisons sorted few ids, more where the ends of runs are many to join.
constexpr int kMinChunk = 16, kMinSortedChunk = 32;
constexpr int64_t kSumWaves = 2048;
// MiB that each sorting kernel clears, by 256 blocks.
constexpr int kEarlyBlocks = 256;
constexpr int64_t kEarlyRank = 40, kEarlyCount = 20, kEarlyPlace = 40;
constexpr int64_t kMaxBlocks = 1 << 20;  // a launch holds fewer than 2^32 threads; blocks take several shares beyond
// Up to so many tiles every block adds up the tiles before its own by itself;
// more are scanned by a kernel between.
constexpr int32_t kScanTiles = 32;

struct Sort {
    uint2 *ids[2];        // (row, row of grad_out) of each id, before and after a pass
    uint32_t *cnt, *tot;  // [tile][bin], [bin]
    uint32_t *ccnt;       // rows form: runs that begin in a chunk's tile before it
    uint32_t *hcnt;       // rows form: runs that begin in each tile
    float *part;          // [chunk][2][dim]: sums of runs that began before / go on behind the chunk
    int64_t n;
    int32_t ntiles, digit;
    uint32_t none;        // key of ids without a row: the number of rows, sorted last
};

// Rows of a gradient that is overwritten, as bytes: zero is the same in every type.
struct Rows {
    char *data;
    int64_t stride, bytes;  // from row to row, of a row
    int64_t r0, r1;         // of a kernel that clears rows unseen: which ones
};

// Clears the rows [r0, r1) that taken(r) leaves, by a block of BLOCK threads, a wave on a row at most.  HOW: past the
// caches beside other work (325 us for the batch of 65,536 ids, 354 through them), through them where clearing is most
// of the kernel (four ids, 128,000 x 4,096 bf16: 181 us, 193 past them; 1,000,000 x 64 fp32: 37, 53).
template <int BLOCK, int HOW, typename Taken>
__device__ __forceinline__ void clear_rows(const Rows &g, int64_t r0, int64_t r1, Taken taken) {
    constexpr int V = 8;  // 16 bytes, aligned to two
    const float zero[V] = {};
    const int64_t nv = (g.bytes / 2 + V - 1) / V;
    int tz = 64;  // threads side by side on a row
    while (tz > 1 && tz / 2 >= nv) tz >>= 1;
    const int x = threadIdx.x & (tz - 1);
    for (int64_t r = r0 + threadIdx.x / tz; r < r1; r += BLOCK / tz) {
        if (taken(r)) continue;
        _Float16 *row = reinterpret_cast<_Float16 *>(g.data + r * g.stride);
        for (int64_t at = x * V; at < g.bytes / 2; at += tz * V) store_vec<_Float16, V, HOW>(row + at, (int32_t)(g.bytes / 2 - at), zero);
    }
}

// Sorting leaves most CUs and all of HBM idle, so its kernels have more blocks, from number `first` on, that clear rows
// whatever ids name them: the sums are written later.  (65,536 ids, 128,000 x 4,096 bf16: 336 us, 326 so;
// 3,000 ids, 50,000 x 1,024: 32.1, 29.0.)
__device__ __forceinline__ bool cleared_early(const Rows &g, int first) {
    if ((int)blockIdx.x < first) return false;
    const int64_t blocks = gridDim.x - first, per = (g.r1 - g.r0 + blocks - 1) / blocks;
    const int64_t r0 = g.r0 + ((int)blockIdx.x - first) * per;
    clear_rows<kSortBlock, STREAM>(g, r0, min(r0 + per, g.r1), [](int64_t) { return false; });
    return true;
}

// The rows that N ids name, none for those without one; at(k): the place of the k-th of them, none behind the last id.
// Places behind the last are read as the last: the loads have no branches between them and are in flight together.
template <int N, typename At>
__device__ __forceinline__ void load_keys(const GradCall &c, uint32_t none, At at, uint32_t (&key)[N]) {
    int64_t id[N];
    if (c.tok.index_type == RECMG_I32) {
#pragma unroll
        for (int k = 0; k < N; ++k) id[k] = static_cast<const int32_t *>(c.tok.ids)[min((int64_t)at(k), c.tok.n - 1)];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) id[k] = static_cast<const int64_t *>(c.tok.ids)[min((int64_t)at(k), c.tok.n - 1)];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t r = id[k] == c.padding_token ? -1 : local_row(id[k], c.tok.first_row, c.tok.rows);
        key[k] = r < 0 || at(k) >= c.tok.n ? none : (uint32_t)r;
    }
}

// The bag of position p of the batch: the last that begins at or before it (bag 0 for positions before them all).
__device__ __forceinline__ int32_t bag_of(const int64_t *offsets, int64_t bags, int64_t p) {
    int64_t lo = 0, hi = bags - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (offsets[mid] <= p) lo = mid;
        else hi = mid - 1;
    }
    return (int32_t)lo;
}

// Up to kRankIds ids: the place of each among the sorted ones is the number of ids that are smaller, or equal and
// earlier.  Every block holds all keys in LDS and places T ids; 64 / T lanes of each wave share one of them, each
// comparing it with a part of the keys.  All CUs take part, and there are n * n comparisons of two or three instructions each:
// less than the barriers and launches of a radix sort.  (A thread's loads of the keys, up to eight, wait for one another.)
__global__ __launch_bounds__(kSortBlock) void k_rank(Sort s, GradCall c, int log_t, Rows early) {
    __shared__ uint4 keys4[kRankIds / 4];
    __shared__ uint32_t cnt[kSortWaves][64];
    uint32_t *keys = reinterpret_cast<uint32_t *>(keys4);
    const int tid = threadIdx.x, t = 1 << log_t, n = (int)s.n;
    if (cleared_early(early, (n + t - 1) >> log_t)) return;
    const int64_t p0 = c.offsets ? c.offsets[0] : 0, pend = c.offsets ? c.offsets[c.num_bags] : 0;
#pragma unroll
    for (int k = 0; k < kRankIds / kSortBlock; ++k) {
        const int j = k * kSortBlock + tid;
        uint32_t key[1] = {~0u};  // behind the ids: not below any
        if (j < n) {
            load_keys<1>(c, s.none, [&](int) { return (int64_t)j; }, key);
            if (c.offsets && p0 + j >= pend) key[0] = s.none;
        }
        keys[j] = key[0];
    }
    const int i = (int)blockIdx.x * t + (tid & (t - 1));
    int32_t pay = i;
    if (c.offsets && tid < t && i < n) pay = bag_of(c.offsets, c.num_bags, p0 + i);
    __syncthreads();
    const uint32_t ki = i < n ? keys[i] : 0u;
    // groups of 4 keys, taken in turn; those before the id's own count equal keys, those behind do not
    const int groups = (n + 3) / 4;
    uint32_t below = 0;
    for (int g = tid >> log_t; g < groups; g += kSortBlock >> log_t) {
        const uint4 k = keys4[g];
        const uint32_t bound = ki + (g < i / 4 ? 1u : 0u);
        below += (uint32_t)(k.x < bound) + (uint32_t)(k.y < bound) + (uint32_t)(k.z < bound) + (uint32_t)(k.w < bound);
    }
    for (int d = t; d < 64; d <<= 1) below += (uint32_t)__shfl_xor((int)below, d, 64);
    if ((tid & 63) < t) cnt[tid >> 6][tid & 63] = below;
    __syncthreads();
    if (tid >= t || i >= n) return;
    for (int k = 1; k < kSortWaves; ++k) below += cnt[k][tid];
    for (int j = i & ~3; j < i; ++j) below += keys[j] == ki ? 1u : 0u;  // equal and earlier in the id's own group
    s.ids[0][below] = make_uint2(ki, (uint32_t)pay);
}

// How many of the n offsets are not behind position p[0], and p[1], by the whole block: rounds of 1,024 probes at once.
__device__ __forceinline__ void offsets_up_to(const int64_t *offsets, int64_t n, const int64_t (&p)[2], int64_t (&upto)[2]) {
    int64_t lo[2] = {0, 0}, hi[2] = {n, n};  // the answers lie in [lo, hi]
    while (hi[0] > lo[0] || hi[1] > lo[1]) {
        int64_t step[2];
        bool below[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            step[q] = (hi[q] - lo[q] + kSortBlock - 1) / kSortBlock;
            const int64_t at = lo[q] + threadIdx.x * step[q];
            below[q] = at < hi[q] && offsets[at] <= p[q];
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t k = __syncthreads_count(below[q]);
            if (hi[q] == lo[q]) continue;
            hi[q] = k == 0 ? lo[q] : min(hi[q], lo[q] + k * step[q]);
            if (k > 0) lo[q] += (k - 1) * step[q] + 1;
        }
    }
    upto[0] = lo[0];
    upto[1] = lo[1];
}

// One more of digit d (valid lanes), in LDS.  Where a wave's digits are all the same, as in a run of a frequent token,
// one lane counts them: 64 additions to one word would queue.
__device__ __forceinline__ void count_digit(uint32_t *hist, bool valid, uint32_t d) {
    const unsigned long long all = __ballot(valid);
    if (!valid) return;
    const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)d);
    if (__ballot(d == first) == all) {
        if ((int)(threadIdx.x & 63) == __ffsll(all) - 1) atomicAdd(&hist[first], (uint32_t)__popcll(all));
    } else {
        atomicAdd(&hist[d], 1u);
    }
}

// Exclusive scan over the 1,024 threads; tmp: LDS, kSortWaves entries, not in use by other waves when called.
__device__ __forceinline__ uint32_t sort_scan(uint32_t v, uint32_t *tmp, uint32_t *total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t upto = (uint32_t)wave_incl_scan((int)v);
    if (lane == 63) tmp[w] = upto;
    __syncthreads();
    uint32_t sums[kSortWaves], before = 0, all = 0;  // read together
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) sums[k] = tmp[k];
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
        before += k < w ? sums[k] : 0u;
        all += sums[k];
    }
    *total = all;
    return before + upto - v;
}

// Row and grad_out row of each id; digits of the first pass counted.
// A thread takes consecutive ids.  The bag of an id is the number of bags that begin up to it, less one: the beginnings
// in the tile are marked in LDS and added up (a search per id took 5 us of the kernel's 10 for 81,920 ids in 2,048 bags).
__global__ __launch_bounds__(kSortBlock) void k_sort_start(Sort s, GradCall c, Rows early) {
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t begun[kSortTile];
    __shared__ uint32_t tmp[kSortWaves];
    const int tid = threadIdx.x, bins = 1 << s.digit;
    if (cleared_early(early, s.ntiles)) return;
    for (int d = tid; d < bins; d += kSortBlock) hist[d] = 0;
    const int64_t i0 = (int64_t)blockIdx.x * kSortTile + tid * kKeysPerThread;
    uint32_t key[kKeysPerThread];
    int32_t pay[kKeysPerThread];
    load_keys<kKeysPerThread>(c, s.none, [&](int k) { return i0 + k; }, key);
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) pay[k] = (int32_t)(i0 + k);
    if (c.offsets) {
        const int64_t p = c.offsets[0] + (int64_t)blockIdx.x * kSortTile, pend = c.offsets[c.num_bags];
#pragma unroll
        for (int k = 0; k < kKeysPerThread; ++k) begun[tid * kKeysPerThread + k] = 0;
        int64_t b0 = 0, b1 = c.num_bags;  // the bags to look at; those before b0 begin before the tile
        if (c.num_bags > kSortTile) {
            const int64_t q[2] = {p, p + kSortTile - 1};
            int64_t upto[2];
            offsets_up_to(c.offsets, c.num_bags, q, upto);
            b0 = upto[0];
            b1 = upto[1];
        }
        __syncthreads();
        uint32_t before = 0;
        for (int64_t b = b0 + tid; b < b1; b += kSortBlock) {
            const int64_t at = c.offsets[b] - p;
            if (at <= 0) ++before;
            else if (at < kSortTile) atomicAdd(&begun[at], 1u);
        }
        uint32_t earlier;
        sort_scan(before, tmp, &earlier);
        __syncthreads();
        uint32_t run = 0;
#pragma unroll
        for (int k = 0; k < kKeysPerThread; ++k) {
            run += begun[tid * kKeysPerThread + k];
            pay[k] = (int32_t)run;
        }
        uint32_t all;
        const int32_t bag = (int32_t)(b0 + earlier + sort_scan(run, tmp, &all)) - 1;  // offsets[0] counts: never below 0
#pragma unroll
        for (int k = 0; k < kKeysPerThread; ++k) {
            pay[k] = max(0, min((int32_t)(c.num_bags - 1), bag + pay[k]));  // offsets that do not rise: some bag
            if (p + tid * kKeysPerThread + k >= pend) key[k] = s.none;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        if (i0 + k < s.n) s.ids[0][i0 + k] = make_uint2(key[k], (uint32_t)pay[k]);
        count_digit(hist, i0 + k < s.n, key[k] & (bins - 1));
    }
    __syncthreads();
    for (int d = tid; d < bins; d += kSortBlock) s.cnt[(int64_t)blockIdx.x * bins + d] = hist[d];
}

// Digits of a later pass, tile by tile.  (Counted by the pass before, as it places the ids, it took that pass 55 us
// instead of 9: the atomics on a frequent row's counter queue up in memory.)
__global__ __launch_bounds__(kSortBlock) void k_sort_count(Sort s, int from, int shift, Rows early) {
    __shared__ uint32_t hist[kBins];
    const int tid = threadIdx.x, bins = 1 << s.digit;
    if (cleared_early(early, s.ntiles)) return;
    for (int d = tid; d < bins; d += kSortBlock) hist[d] = 0;
    __syncthreads();
    uint32_t key[kKeysPerThread];
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const int64_t i = (int64_t)blockIdx.x * kSortTile + k * kSortBlock + tid;
        key[k] = i < s.n ? s.ids[from][i].x : 0u;
    }
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k)
        count_digit(hist, (int64_t)blockIdx.x * kSortTile + k * kSortBlock + tid < s.n, (key[k] >> shift) & (bins - 1));
    __syncthreads();
    for (int d = tid; d < bins; d += kSortBlock) s.cnt[(int64_t)blockIdx.x * bins + d] = hist[d];
}

// Columns of cnt[tile][bin] made exclusive sums over the tiles, their totals in tot.  A block takes 64 bins, its 16
// waves consecutive parts of the tiles.
__global__ __launch_bounds__(kSortBlock) void k_scan_tiles(uint32_t *cnt, uint32_t *tot, int32_t ntiles, int32_t bins) {
    __shared__ uint32_t sums[kSortWaves][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int32_t d = (int32_t)blockIdx.x * 64 + lane;
    const int32_t per = (ntiles + kSortWaves - 1) / kSortWaves;
    const int32_t t0 = min(w * per, ntiles), t1 = min(t0 + per, ntiles);
    uint32_t sum = 0;
    if (d < bins)
        for (int32_t t = t0; t < t1; ++t) sum += cnt[(int64_t)t * bins + d];
    sums[w][lane] = sum;
    __syncthreads();
    uint32_t run = 0, all = 0;
    for (int k = 0; k < kSortWaves; ++k) {
        if (k < w) run += sums[k][lane];
        all += sums[k][lane];
    }
    if (d >= bins) return;
    for (int32_t t = t0; t < t1; ++t) {
        const uint32_t v = cnt[(int64_t)t * bins + d];
        cnt[(int64_t)t * bins + d] = run;
        run += v;
    }
    if (w == 0) tot[d] = all;
}

// One tile's ids to their places by one digit.
__global__ __launch_bounds__(kSortBlock) void k_sort_place(Sort s, int from, int shift, int scanned, Rows early) {
    __shared__ uint32_t wcnt[kSortWaves][kBins];
    __shared__ uint32_t base[kBins];
    __shared__ uint32_t tmp[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bins = 1 << s.digit;
    if (cleared_early(early, s.ntiles)) return;
    const int32_t tile = blockIdx.x;
    const int64_t i0 = (int64_t)tile * kSortTile + w * kWaveKeys + lane;
    uint2 id[kKeysPerThread];
    uint32_t rank[kKeysPerThread];
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) id[k] = i0 + k * 64 < s.n ? s.ids[from][i0 + k * 64] : make_uint2(0, 0);
    for (int d = lane; d < bins; d += 64) wcnt[w][d] = 0;
    // places of the tile's first id of each digit (the scan's sums wrap only where n does: never)
    uint32_t before = 0, total = 0;
    if (tid < bins) {
        if (scanned) {
            before = s.cnt[(int64_t)tile * bins + tid];
            total = s.tot[tid];
        } else {
            uint32_t v[kScanTiles];  // all in flight together
#pragma unroll
            for (int t = 0; t < kScanTiles; ++t) v[t] = t < s.ntiles ? s.cnt[(int64_t)t * bins + tid] : 0u;
#pragma unroll
            for (int t = 0; t < kScanTiles; ++t) {
                before += t < tile ? v[t] : 0u;
                total += v[t];
            }
        }
    }
    uint32_t all;
    const uint32_t smaller = sort_scan(total, tmp, &all);
    if (tid < bins) base[tid] = smaller + before;
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const bool valid = i0 + k * 64 < s.n;
        const uint32_t d = (id[k].x >> shift) & (bins - 1);
        unsigned long long same = __ballot(valid);
        for (int b = 0; b < s.digit; ++b) {
            const bool bit = (d >> b) & 1;
            const unsigned long long m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        // the lowest lane of each digit counts all of them; one wave's LDS operations stay in order
        const int leader = valid ? __ffsll((unsigned long long)same) - 1 : lane;
        uint32_t old = 0;
        if (valid && leader == lane) old = atomicAdd(&wcnt[w][d], (uint32_t)__popcll(same));
        old = (uint32_t)__shfl((int)old, leader, 64);
        rank[k] = old + (uint32_t)__popcll(same & ((1ull << lane) - 1));
    }
    __syncthreads();
    if (tid < bins) {
        uint32_t run = base[tid], v[kSortWaves];
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) v[k] = wcnt[k][tid];
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            wcnt[k][tid] = run;
            run += v[k];
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        if (i0 + k * 64 >= s.n) break;
        const uint32_t to = wcnt[w][(id[k].x >> shift) & (bins - 1)] + rank[k];
        s.ids[from ^ 1][to] = id[k];
    }
}

// Rows form: runs that begin in each tile, and in a tile before each of its chunks.
__global__ __launch_bounds__(kSortBlock) void k_runs(Sort s, int at, int32_t chunk) {
    __shared__ int tmp[16];
    const int64_t i0 = (int64_t)blockIdx.x * kSortTile + (int64_t)threadIdx.x * kKeysPerThread;
    const uint2 *ids = s.ids[at];
    int own = 0;
    uint32_t prev = i0 > 0 && i0 <= s.n ? ids[i0 - 1].x : s.none;
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const uint32_t v = i0 + k < s.n ? ids[i0 + k].x : s.none;
        own += v < s.none && (i0 + k == 0 || v != prev);
        prev = v;
    }
    int all;
    const int before = block_excl_scan(own, tmp, &all);
    static_assert(kMinChunk % kKeysPerThread == 0, "chunks begin at a thread's first id");
    if (i0 % chunk == 0 && i0 < s.n) s.ccnt[i0 / chunk] = (uint32_t)before;
    if (threadIdx.x == 0) s.hcnt[blockIdx.x] = (uint32_t)all;
}

// How the rows form knows the runs before a chunk: whole-table gradients need not; by counting them in the sorted ids
// (few ids); from the counts of chunks and tiles, the tiles added up here or by k_scan_tiles.
enum { RUNS_NONE = 0, RUNS_COUNT = 1, RUNS_TILES = 2, RUNS_SCANNED = 3 };

struct SumArgs {
    int64_t nchunk, zero_blocks;
    int32_t chunk, slices, runs, zero_rows;  // zero_rows: rows that a clearing block takes
};

// Runs that begin in the ids [p0, p1), counted by the whole block; tmp: LDS, blockDim.x / 64 entries.
__device__ __forceinline__ int count_runs(const Sort &s, const uint2 *ids, int p0, int p1, int *tmp) {
    constexpr int U = 8;
    int own = 0;
    for (int q = p0 + (int)threadIdx.x; q < p1; q += U * (int)blockDim.x) {
        uint32_t k[U], before[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = q + u * (int)blockDim.x;
            k[u] = p < p1 ? ids[p].x : s.none;
            before[u] = p < p1 && p > 0 ? ids[p - 1].x : s.none;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) own += k[u] < s.none && k[u] != before[u];
    }
    own = wave_sum(own);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = own;
    __syncthreads();
    int all = 0;
    for (int k = 0; k < (int)(blockDim.x >> 6); ++k) all += tmp[k];
    __syncthreads();
    return all;
}

// Runs that begin before a chunk (RUNS_TILES and RUNS_SCANNED).  Every lane of the wave calls, each with a chunk.
__device__ __forceinline__ int64_t runs_before(const Sort &s, const SumArgs &a, int64_t chunk) {
    const int32_t tile = (int32_t)(chunk * a.chunk / kSortTile);
    if (a.runs == RUNS_SCANNED) return (int64_t)s.hcnt[tile] + s.ccnt[chunk];
    static_assert(kScanTiles <= 64, "a lane per tile");
    const int lane = threadIdx.x & 63;
    const int upto = wave_incl_scan(lane < s.ntiles ? (int)s.hcnt[lane] : 0);
    const int before = __shfl(upto, tile > 0 ? tile - 1 : 0, 64);
    return (int64_t)(tile > 0 ? before : 0) + s.ccnt[chunk];
}

// Where a run's sum goes, and the old value for a gradient that is added to.
template <int WT, int V>
__device__ __forceinline__ void write_row(const GradCall &c, int64_t row, int32_t col, int32_t left, const float (&acc)[V]) {
    elem_t<WT> *dst = static_cast<elem_t<WT> *>(c.grad) + row * c.grad_stride + col;
    float y[V];
#pragma unroll
    for (int v = 0; v < V; ++v) y[v] = acc[v] * c.scale;
    if (left <= 0) return;
    if (c.accumulate) {
        float old[V];
        load_vec<elem_t<WT>, V>(dst, left, old);
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] += old[v];
    }
    store_vec<elem_t<WT>, V>(dst, left, y);
}

template <int V>
__device__ __forceinline__ void write_part(const Sort &s, int32_t dim, int64_t chunk, int which, int32_t col, int32_t left,
                                           const float (&acc)[V]) {
    if (left > 0) store_vec<float, V>(s.part + (chunk * 2 + which) * dim + col, left, acc);
}

// One value of a group of LANES lanes (u the same in all of them).
template <int LANES>
__device__ __forceinline__ int group_read(int v, int u) {
    if constexpr (LANES == 64) return __builtin_amdgcn_readlane(v, u);
    else return __shfl(v, u, LANES);
}

// The first of the n sorted keys that is not below k.
__device__ __forceinline__ int64_t first_not_below(const uint2 *ids, int64_t n, uint32_t k) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (ids[mid].x < k) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// U rows of grad_out in flight per group: four, in 2,048 waves, for 65,536 ids of 4,096 bf16 columns (2, 4, 8 rows in 4,096
// waves: 356, 360, 373 us; in 2,048: 334, 333, 378; in 1,024: 406, 338); eight where rows are short.
template <int GT, int WT, int V, int LANES>
__global__ __launch_bounds__(kSumBlock) void k_sum(Sort s, GradCall c, SumArgs a, Rows rest, int at) {
    constexpr int kGroups = kSumBlock / LANES, U = LANES == 64 ? 4 : 8;
    __shared__ int tmp[kSumBlock / 64];
    __shared__ uint32_t there[kMaxZeroRows / 32];
    const uint2 *ids = s.ids[at];
    const int64_t sum_blocks = (int64_t)gridDim.x - a.zero_blocks;
    const int64_t block = blockIdx.x;
    if (block >= sum_blocks) {
        for (int64_t r0 = rest.r0 + (block - sum_blocks) * a.zero_rows; r0 < rest.r1; r0 += a.zero_blocks * a.zero_rows) {
            const int64_t r1 = min(r0 + a.zero_rows, rest.r1);
            if (threadIdx.x < kMaxZeroRows / 32) there[threadIdx.x] = 0;
            __syncthreads();
            for (int64_t r = r0 + threadIdx.x; r < r1; r += kSumBlock) {  // a binary search per row, side by side
                const int64_t p = first_not_below(ids, s.n, (uint32_t)r);
                if (p < s.n && ids[p].x == (uint32_t)r) atomicOr(&there[(r - r0) >> 5], 1u << ((r - r0) & 31));
            }
            __syncthreads();
            clear_rows<kSumBlock, STREAM>(rest, r0, r1, [&](int64_t r) { return there[(r - r0) >> 5] >> ((r - r0) & 31) & 1; });
            __syncthreads();
        }
        return;
    }
    const int sub = threadIdx.x & (LANES - 1);
    const elem_t<GT> *g = static_cast<const elem_t<GT> *>(c.grad_out);
    const unsigned long long lanes = LANES == 64 ? ~0ull : (1ull << LANES) - 1;
    const int shift = threadIdx.x & 63 & ~(LANES - 1);  // the group's first lane of its wave
    // the whole block goes round together: RUNS_COUNT has barriers
    for (int64_t group0 = block * kGroups; group0 < a.nchunk * a.slices; group0 += sum_blocks * kGroups) {
        const int64_t group = group0 + threadIdx.x / LANES;
        const int64_t chunk = min(group / a.slices, a.nchunk - 1);
        const int32_t slice = (int32_t)(group - group / a.slices * a.slices);
        const int64_t p0 = chunk * a.chunk, p1 = min(p0 + a.chunk, s.n);
        int64_t base = 0;
        if (a.runs == RUNS_COUNT) {
            const int first = (int)(group0 / a.slices * a.chunk);
            base = count_runs(s, ids, 0, first, tmp);
            int more = 0;  // from the block's first chunk to the group's
            for (int p = first + sub; p < (int)p0; p += LANES) more += ids[p].x < s.none && (p == 0 || ids[p].x != ids[p - 1].x);
#pragma unroll
            for (int d = LANES / 2; d >= 1; d >>= 1) more += __shfl_xor(more, d, LANES);
            base += more;
        } else if (a.runs != RUNS_NONE) {
            base = runs_before(s, a, chunk);
        }
        if (group >= a.nchunk * a.slices) continue;
        const int32_t col = (slice * LANES + sub) * V, left = c.dim - col;
        const uint32_t last = p0 > 0 ? ids[p0 - 1].x : s.none;
        uint32_t cur = s.none;  // the run being summed, its row in grad, whether it began in this chunk
        int64_t row = 0;
        bool begun = true;
        float acc[V];
        int64_t done = p0;
        for (int64_t b = p0; b < p1; b += LANES) {
            const int64_t p = b + sub;
            const uint2 id = p < p1 ? ids[p] : make_uint2(s.none, 0);
            const uint32_t kl = id.x;
            const int32_t pl = (int32_t)id.y;
            const int nv = __popcll((__ballot(kl < s.none) >> shift) & lanes);  // ids without a row come last
            int32_t rl = 0;  // rows form: the run's number, less base
            if (a.runs != RUNS_NONE) {
                const bool head = sub < nv && (p == 0 || ids[p - 1].x != kl);
                const unsigned long long heads = (__ballot(head) >> shift) & lanes;
                rl = __popcll(heads & ((2ull << sub) - 1)) - 1;
                if (slice == 0 && sub < nv) {
                    // the lane of a run's first id names its row, that of the last id the number of rows
                    if (head) c.rows_out[base + rl] = (int32_t)kl;
                    if (p + 1 == s.n || ids[p + 1].x == s.none) *c.count = base + rl + 1;
                }
                if (slice == 0 && p == 0 && kl == s.none) *c.count = 0;
            }
            for (int u0 = 0; u0 < nv; u0 += U) {
                float x[U][V];
                uint32_t ku[U];
                int32_t ru[U];
                int64_t pay[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int from = min(u0 + u, nv - 1);
                    ku[u] = (uint32_t)group_read<LANES>((int)kl, from);
                    ru[u] = a.runs != RUNS_NONE ? group_read<LANES>(rl, from) : 0;
                    pay[u] = group_read<LANES>(pl, from);
                }
                load_vecs<elem_t<GT>, V, U>(c.dim % V == 0, left, [&](int u) { return g + pay[u] * c.grad_out_stride + col; }, x);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (u0 + u >= nv) break;
                    if (ku[u] != cur) {
                        if (cur != s.none) {
                            if (begun) write_row<WT, V>(c, row, col, left, acc);
                            else write_part<V>(s, c.dim, chunk, 0, col, left, acc);
                        }
                        begun = cur != s.none || ku[u] != last;
                        cur = ku[u];
                        row = a.runs != RUNS_NONE ? base + ru[u] : (int64_t)cur;
#pragma unroll
                        for (int v = 0; v < V; ++v) acc[v] = 0.f;
                    }
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[v] += x[u][v];
                }
            }
            if (a.runs != RUNS_NONE && nv > 0) base += group_read<LANES>(rl, nv - 1) + 1;
            done = b + nv;
            if (nv < LANES) break;
        }
        if (cur == s.none) continue;
        const bool goes_on = done == p1 && p1 < s.n && ids[p1].x == cur;
        if (!begun) write_part<V>(s, c.dim, chunk, 0, col, left, acc);
        else if (goes_on) write_part<V>(s, c.dim, chunk, 1, col, left, acc);
        else write_row<WT, V>(c, row, col, left, acc);
    }
}

// Runs over several chunks: the block of the chunk where a run begins adds its parts.  Most blocks find no such run, so
// they are few and small, one per chunk and 1,024 columns: for 1,024 chunks of 4,096 columns they took 24 us, blocks of
// 1,024 threads for 256 columns each 113.  1 << log_tc threads side by side on vectors of 4 columns, the others, where
// the columns are fewer, on every (256 >> log_tc)-th part; their sums meet in LDS, in a fixed order.
template <int WT>
__global__ __launch_bounds__(kSumBlock) void k_join(Sort s, GradCall c, SumArgs a, int at, int log_tc) {
    constexpr int V = 4, U = 8;  // U: parts in flight
    __shared__ float red[kSumBlock * V];
    __shared__ int tmp[kSumBlock / 64];
    const uint2 *ids = s.ids[at];
    const int tc = 1 << log_tc, groups = kSumBlock >> log_tc;
    const int x = threadIdx.x & (tc - 1), y = threadIdx.x >> log_tc;
    const int32_t col = ((int32_t)(blockIdx.y << log_tc) + x) * V, left = c.dim - col;
    for (int64_t chunk = blockIdx.x; chunk + 1 < a.nchunk; chunk += gridDim.x) {
        const int64_t p0 = chunk * a.chunk, p1 = p0 + a.chunk;
        const uint32_t k = ids[p1 - 1].x, next_key = ids[p1].x, first_key = ids[p0].x, last = p0 > 0 ? ids[p0 - 1].x : s.none;
        if (k == s.none || next_key != k || (first_key == k && p0 > 0 && last == k)) continue;
        int64_t end = chunk + 1;  // the last chunk whose first id belongs to the run
        for (;;) {
            const int64_t next = end + 1 + threadIdx.x;
            const int more = __syncthreads_count(next < a.nchunk && ids[next * a.chunk].x == k);
            end += more;
            if (more < kSumBlock) break;
        }
        float acc[V] = {0.f, 0.f, 0.f, 0.f};
        for (int64_t j0 = chunk + y; j0 <= end; j0 += U * groups) {
            float v[U][V];
            load_vecs<float, V, U>(c.dim % V == 0, left, [&](int u) {  // parts behind the last: the last, and not added
                const int64_t j = min(j0 + u * groups, end);
                return s.part + (j * 2 + (j == chunk ? 1 : 0)) * c.dim + col;
            }, v);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j0 + u * groups <= end)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] += v[u][i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) red[threadIdx.x * V + i] = acc[i];
        const int64_t runs = a.runs == RUNS_NONE    ? 0
                             : a.runs == RUNS_COUNT ? count_runs(s, ids, 0, (int)p1, tmp)
                                                    : runs_before(s, a, chunk + 1);
        __syncthreads();
        if (y == 0) {
            const int parts = (int)min((int64_t)groups, end - chunk + 1);
            for (int q = 1; q < parts; ++q)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += red[(q * tc + x) * V + i];
            write_row<WT, V>(c, a.runs != RUNS_NONE ? runs - 1 : (int64_t)k, col, left, acc);
        }
        __syncthreads();
    }
}

// Rows below `bound` that ids name, each counted at its first id: thread t holds the row of id t.  keys4: LDS, a key per
// thread; tmp: LDS, a word per wave.  The whole block calls and gets the number.
template <int BLOCK>
__device__ __forceinline__ int firsts_below(uint32_t key, uint32_t bound, uint4 *keys4, int *tmp) {
    uint32_t *keys = reinterpret_cast<uint32_t *>(keys4);
    const int t = threadIdx.x;
    keys[t] = key;
    __syncthreads();
    bool first = key < bound;
    if (first) {
        bool equal = false;
#pragma unroll 8
        for (int g = 0; g < t / 4; ++g) {
            const uint4 k = keys4[g];
            equal |= k.x == key || k.y == key || k.z == key || k.w == key;
        }
        for (int j = t & ~3; j < t; ++j) equal |= keys[j] == key;
        first = !equal;
    }
    const unsigned long long all = __ballot(first);
    if ((t & 63) == 0) tmp[t >> 6] = __popcll(all);
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int k = 0; k < BLOCK / 64; ++k) sum += tmp[k];
    return sum;
}

// Few ids, no bags.  The block of (id, slice of the columns) looks for equal ids; if none is
// earlier it sums their rows, each wave those of a part of the ids, and the waves' sums meet in LDS.  Further blocks mark
// the ids' rows among theirs in LDS and clear the others.  Rows form (kPer = 1): a block numbers its row by counting the
// rows below it, the first block all of them.
template <int GT, int WT, int kPer>
__global__ __launch_bounds__(kDirectBlock) void k_direct(GradCall c, int32_t slices, Rows rest, int64_t zero_blocks,
                                                         int32_t zero_rows) {
    constexpr int V = 8, kWaves = kDirectBlock / 64;
    __shared__ float red[kWaves][64 * V];
    __shared__ int count[kWaves];
    __shared__ uint32_t there[kMaxZeroRows / 32];
    __shared__ uint4 keys4[kPer == 1 ? kDirectBlock / 4 : 1];  // rows form
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t none = (uint32_t)c.tok.rows;
    const int64_t sum_blocks = (int64_t)gridDim.x - zero_blocks;
    // wave w takes the ids [w * kPer * 64, ...), in order of (k, lane)
    uint32_t key[kPer];
    const int j0 = w * kPer * 64 + lane;
    load_keys<kPer>(c, none, [&](int k) { return (int64_t)(j0 + k * 64); }, key);
    if ((int64_t)blockIdx.x >= sum_blocks) {
        for (int64_t r0 = rest.r0 + (blockIdx.x - sum_blocks) * zero_rows; r0 < rest.r1; r0 += zero_blocks * zero_rows) {
            const int64_t r1 = min(r0 + zero_rows, rest.r1);
            if (threadIdx.x < kMaxZeroRows / 32) there[threadIdx.x] = 0;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (key[k] >= r0 && key[k] < r1) {  // r1 <= rows: never `none`
                    const uint32_t r = key[k] - (uint32_t)r0;
                    atomicOr(&there[r >> 5], 1u << (r & 31));
                }
            __syncthreads();
            clear_rows<kDirectBlock, CACHED>(rest, r0, r1, [&](int64_t r) { return there[(r - r0) >> 5] >> ((r - r0) & 31) & 1; });
            __syncthreads();
        }
        return;
    }
    const int i = (int)(blockIdx.x / slices);
    const int32_t slice = (int32_t)(blockIdx.x - (int64_t)i * slices);
    const int32_t col = (slice * 64 + lane) * V, left = c.dim - col;
    uint32_t own_key[1];
    load_keys<1>(c, none, [&](int) { return (int64_t)i; }, own_key);
    const uint32_t ki = own_key[0];
    if (kPer == 1 && c.rows_out && blockIdx.x == 0) {
        const int all = firsts_below<kDirectBlock>(key[0], none, keys4, count);
        if (threadIdx.x == 0) *c.count = all;
        __syncthreads();
    }
    if (ki == none) return;
    unsigned long long same[kPer];
    int own = 0;
    bool earlier = false;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        same[k] = __ballot(key[k] == ki);
        own += __popcll(same[k]);
        earlier |= key[k] == ki && j0 + k * 64 < i;
    }
    if (lane == 0) count[w] = own;
    if (__syncthreads_or(earlier)) return;  // the first of the equal ids sums them
    int64_t row = (int64_t)ki;
    if (kPer == 1 && c.rows_out) {
        row = firsts_below<kDirectBlock>(key[0], ki, keys4, reinterpret_cast<int *>(red));
        if (slice == 0 && threadIdx.x == 0) c.rows_out[row] = (int32_t)ki;
        __syncthreads();
    }
    const elem_t<GT> *g = static_cast<const elem_t<GT> *>(c.grad_out);
    float acc[V] = {};
    // the rows of the next U ids of the mask, in flight together; behind the last, row i once more, not added
    const auto add = [&](auto un, unsigned long long &m, int64_t j0) {
        constexpr int U = decltype(un)::value;
        float x[U][V];
        bool there_is[U];
        int64_t j[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            there_is[u] = m != 0;
            j[u] = m ? j0 + (__ffsll(m) - 1) : i;
            m &= m - 1;
        }
        load_vecs<elem_t<GT>, V, U>(c.dim % V == 0, left, [&](int u) { return g + j[u] * c.grad_out_stride + col; }, x);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (there_is[u])
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += x[u][v];
    };
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        unsigned long long m = same[k];
        while (m) {
            if (__popcll(m) > 2) add(std::integral_constant<int, 8>(), m, w * kPer * 64 + k * 64);
            else add(std::integral_constant<int, 1>(), m, w * kPer * 64 + k * 64);
        }
    }
    const int mine = i / (kPer * 64);  // the wave that holds id i
    int others = 0;
    for (int k = 0; k < kWaves; ++k) others += k == mine ? 0 : count[k];
    if (others) {  // the same in all waves
#pragma unroll
        for (int v = 0; v < V; ++v) red[w][v * 64 + lane] = acc[v];
        __syncthreads();
        if (w != mine) return;
        for (int k = mine + 1; k < kWaves; ++k)
            if (count[k])
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += red[k][v * 64 + lane];
    }
    if (w == mine) write_row<WT, V>(c, row, col, left, acc);
}

// A gradient without an id.
__global__ __launch_bounds__(kSumBlock) void k_clear(Rows rest, int32_t zero_rows) {
    for (int64_t r0 = rest.r0 + (int64_t)blockIdx.x * zero_rows; r0 < rest.r1; r0 += (int64_t)gridDim.x * zero_rows)
        clear_rows<kSumBlock, CACHED>(rest, r0, min(r0 + zero_rows, rest.r1), [](int64_t) { return false; });
}

__global__ void k_no_rows(int64_t *count) { *count = 0; }

int log2_ceil(int64_t x, int most) {
    int l = 0;
    while (l < most && (int64_t(1) << l) < x) ++l;
    return l;
}

unsigned capped(int64_t blocks) { return (unsigned)(blocks < 1 ? 1 : blocks > kMaxBlocks ? kMaxBlocks : blocks); }

// Rows that a clearing block takes: some 64 KiB, so that the search for its rows costs less than the stores.
int32_t zero_rows_of(const GradCall &c) {
    const int64_t rows = 65536 / ((int64_t)c.dim * elem_size(c.grad_dtype));
    return (int32_t)(rows < 8 ? 8 : rows > kMaxZeroRows ? kMaxZeroRows : rows);
}

template <int GT, int WT>
void sums_typed(const GradCall &c, const Sort &s, SumArgs a, const Rows &rest, int at, Launches &run) {
    constexpr int V = GT == RECMG_F32 && WT == RECMG_F32 ? 4 : 8;
    const int32_t nv = (c.dim + V - 1) / V;
    const int lanes = nv <= 16 ? 16 : nv <= 32 ? 32 : 64;
    a.slices = (nv + lanes - 1) / lanes;
    const unsigned blocks = capped((a.nchunk * a.slices * lanes + kSumBlock - 1) / kSumBlock) + (unsigned)a.zero_blocks;
    if (lanes == 16) run(k_sum<GT, WT, V, 16>, blocks, kSumBlock, s, c, a, rest, at);
    else if (lanes == 32) run(k_sum<GT, WT, V, 32>, blocks, kSumBlock, s, c, a, rest, at);
    else run(k_sum<GT, WT, V, 64>, blocks, kSumBlock, s, c, a, rest, at);
    if (a.nchunk > 1) {
        const int log_tc = log2_ceil((c.dim + 3) / 4, 8);
        const dim3 grid(capped(a.nchunk - 1), (unsigned)((c.dim + (4 << log_tc) - 1) / (4 << log_tc)));
        run(k_join<WT>, grid, kSumBlock, s, c, a, at, log_tc);
    }
}

template <int GT, int WT>
void direct_typed(const GradCall &c, const Rows &rest, int64_t zero_blocks, int32_t zero_rows, Launches &run) {
    const int32_t slices = (c.dim + 64 * 8 - 1) / (64 * 8);
    const unsigned blocks = (unsigned)(c.tok.n * slices + zero_blocks);
    // as few ids per wave as the block's waves hold: a frequent id's rows then spread over all of them
    if (c.tok.n <= kDirectBlock) run(k_direct<GT, WT, 1>, blocks, kDirectBlock, c, slices, rest, zero_blocks, zero_rows);
    else if (c.tok.n <= 2 * kDirectBlock) run(k_direct<GT, WT, 2>, blocks, kDirectBlock, c, slices, rest, zero_blocks, zero_rows);
    else run(k_direct<GT, WT, 4>, blocks, kDirectBlock, c, slices, rest, zero_blocks, zero_rows);
}
static_assert(kDirectIds == 4 * kDirectBlock && kDirectRows <= kDirectBlock, "ids per thread of k_direct");

// Calls f<grad_out's type, grad's type>(args...).
#define RECMG_TYPES(f, c, ...)                                                       \
    switch ((c).grad_out_dtype * 3 + (c).grad_dtype) {                               \
        case 0: f<0, 0>(__VA_ARGS__); break;                                         \
        case 1: f<0, 1>(__VA_ARGS__); break;                                         \
        case 2: f<0, 2>(__VA_ARGS__); break;                                         \
        case 3: f<1, 0>(__VA_ARGS__); break;                                         \
        case 4: f<1, 1>(__VA_ARGS__); break;                                         \
        case 5: f<1, 2>(__VA_ARGS__); break;                                         \
        case 6: f<2, 0>(__VA_ARGS__); break;                                         \
        case 7: f<2, 1>(__VA_ARGS__); break;                                         \
        default: f<2, 2>(__VA_ARGS__);                                               \
    }

size_t take(size_t *at, size_t bytes) {
    const size_t here = *at;
    *at += (bytes + 255) & ~size_t(255);
    return here;
}

}  // namespace

GradPlan grad_plan(int64_t rows, int32_t dim, int64_t n, bool rows_form, bool bags) {
    GradPlan p{};
    if (n == 0) return p;
    p.direct = !bags && (rows_form ? n <= kDirectRows && n * n * dim <= kDirectRowsWork
                                   : n <= kDirectIds && n * dim <= (n <= kDirectFew ? kDirectValuesFew : kDirectValues));
    if (p.direct) return p;
    p.ranked = n <= kRankIds;
    p.ntiles = (int32_t)((n + kSortTile - 1) / kSortTile);
    int bits = 1;
    while (rows >> bits) ++bits;  // the key of ids without a row is `rows` itself
    p.passes = p.ranked ? 0 : (bits + kMaxDigit - 1) / kMaxDigit;
    p.digit = p.ranked ? 0 : (bits + p.passes - 1) / p.passes;
    // chunks: short ones while there are few ids, longer ones, whose ends cost less, beyond: waves of 512 columns
    // (kSumWaves of them at most) that have as many loads in flight as HBM takes well
    p.chunk = p.ranked ? kMinChunk : kMinSortedChunk;
    while (p.chunk < 512 && n * dim / 512 / p.chunk > kSumWaves) p.chunk *= 2;
    p.nchunk = (n + p.chunk - 1) / p.chunk;
    // room for the chunks of any smaller number of ids too
    const int64_t least = (n + kMinChunk - 1) / kMinChunk, full = 512 * (kSumWaves + 1) / dim + 2, longest = (n + 511) / 512;
    const int64_t room = longest > (least < full ? least : full) ? longest : (least < full ? least : full);
    for (int k = 0; k < (p.ranked ? 1 : 2); ++k) p.ids[k] = take(&p.total, n * 8);
    if (!p.ranked) {
        p.cnt = take(&p.total, ((size_t)p.ntiles << p.digit) * 4);
        p.tot = take(&p.total, (size_t)kBins * 4);
        p.ccnt = take(&p.total, rows_form ? (size_t)room * 4 : 0);
        p.hcnt = take(&p.total, rows_form ? (size_t)p.ntiles * 4 : 0);
    }
    p.part = take(&p.total, (size_t)room * 2 * dim * 4);
    return p;
}

void launch_row_gradient(const GradCall &c, const GradPlan &p, char *ws, Launches &run) {
    const bool rows_form = c.rows_out != nullptr;
    const bool fill = !rows_form && !c.accumulate;
    const int32_t zero_rows = fill ? zero_rows_of(c) : 1;
    const int64_t esz = elem_size(c.grad_dtype);
    Rows rest{static_cast<char *>(c.grad), c.grad_stride * esz, c.dim * esz, 0, fill ? c.tok.rows : 0};
    const auto zero_blocks = [&] { return rest.r1 > rest.r0 ? (int64_t)capped((rest.r1 - rest.r0 + zero_rows - 1) / zero_rows) : 0; };
    if (c.tok.n == 0) {
        if (rows_form) run(k_no_rows, 1, 1, c.count);
        else if (fill) run(k_clear, (unsigned)zero_blocks(), kSumBlock, rest, zero_rows);
        return;
    }
    if (p.direct) {
        RECMG_TYPES(direct_typed, c, c, rest, zero_blocks(), zero_rows, run)
        return;
    }
    // the next rows that a sorting kernel clears: as many as take HBM about as long as the kernel takes anyway
    const auto early = [&](int64_t mbytes, int *blocks) {
        Rows r = rest;
        const int64_t rows = (mbytes << 20) / rest.bytes;
        r.r1 = rest.r0 = rest.r1 - rest.r0 < rows ? rest.r1 : rest.r0 + rows;
        *blocks = (int)(r.r1 - r.r0 < kEarlyBlocks ? r.r1 - r.r0 : kEarlyBlocks);
        return r;
    };
    int more = 0;
    Sort s{};
    for (int k = 0; k < 2; ++k) s.ids[k] = reinterpret_cast<uint2 *>(ws + p.ids[k]);
    s.cnt = reinterpret_cast<uint32_t *>(ws + p.cnt);
    s.tot = reinterpret_cast<uint32_t *>(ws + p.tot);
    s.ccnt = reinterpret_cast<uint32_t *>(ws + p.ccnt);
    s.hcnt = reinterpret_cast<uint32_t *>(ws + p.hcnt);
    s.part = reinterpret_cast<float *>(ws + p.part);
    s.n = c.tok.n;
    s.ntiles = p.ntiles;
    s.digit = p.digit;
    s.none = (uint32_t)c.tok.rows;
    SumArgs a{p.nchunk, 0, p.chunk, 0, RUNS_NONE, zero_rows};
    if (p.ranked) {
        const int log_t = c.tok.n <= 2048 ? 3 : 4;  // 512 blocks at most, two on a CU
        const Rows r = early(kEarlyRank, &more);
        run(k_rank, (unsigned)((c.tok.n + (1 << log_t) - 1) >> log_t) + more, kSortBlock, s, c, log_t, r);
        if (rows_form) a.runs = RUNS_COUNT;
    } else {
        const bool scanned = p.ntiles > kScanTiles;
        const int bins = 1 << p.digit;
        Rows r = early(kEarlyCount, &more);
        run(k_sort_start, p.ntiles + more, kSortBlock, s, c, r);
        for (int q = 0; q < p.passes; ++q) {
            if (q > 0) {
                r = early(kEarlyCount, &more);
                run(k_sort_count, p.ntiles + more, kSortBlock, s, q & 1, q * p.digit, r);
            }
            if (scanned) run(k_scan_tiles, (bins + 63) / 64, kSortBlock, s.cnt, s.tot, p.ntiles, bins);
            r = early(kEarlyPlace, &more);
            run(k_sort_place, p.ntiles + more, kSortBlock, s, q & 1, q * p.digit, scanned, r);
        }
        if (rows_form) {
            run(k_runs, p.ntiles, kSortBlock, s, p.passes & 1, p.chunk);
            if (scanned) run(k_scan_tiles, 1, kSortBlock, s.hcnt, s.tot, p.ntiles, 1);
            a.runs = scanned ? RUNS_SCANNED : RUNS_TILES;
        }
    }
    a.zero_blocks = zero_blocks();
    RECMG_TYPES(sums_typed, c, c, s, a, rest, p.passes & 1, run)
}

}  // namespace recmg
