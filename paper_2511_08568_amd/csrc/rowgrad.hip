// Gradient of a lookup with respect to the table's rows:
//   grad[r, :] = scale * sum over the ids i that name row r of grad_out[bag(i), :].
//
// The ids are sorted by row, stably, with the row of grad_out that each stands
// for; equal ids then lie side by side, and each run of them is summed in fp32
// in the order of the ids.  No value is added to by an atomic, so the result is
// the same from call to call.
//
// Sort: radix passes of at most 10 bits over tiles of 4,096 ids: count the
// digits of each tile, then place each id behind the smaller digits, the same
// digit in earlier tiles, earlier waves and earlier lanes.
// Sums: the sorted ids are cut into chunks of equal length whatever the runs, so
// a token that a tenth of a batch repeats takes no longer than others.  A group
// of lanes sums a chunk's runs for one slice of the columns; a run that lies in
// one chunk goes straight to its row, the ends of the others to fp32 partial
// sums that one more kernel adds up.
#include "embedding.h"
#include "recmg_device.h"
#include "values.h"

namespace recmg {

namespace {

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64, kKeysPerThread = kSortTile / kSortBlock;
constexpr int kWaveKeys = kSortTile / kSortWaves;  // consecutive ids of one wave
constexpr int kBins = 1 << kMaxDigit;
constexpr int kSumBlock = 256;
constexpr int64_t kMaxBlocks = 1 << 20;  // a launch holds fewer than 2^32 threads; blocks take several shares beyond
// Up to so many tiles every block adds up the tiles before its own by itself;
// more are scanned by a kernel between.
constexpr int32_t kScanTiles = 32;

struct Sort {
    uint32_t *key[2];
    int32_t *pay[2];
    uint32_t *cnt, *tot;  // [tile][bin], [bin]
    uint32_t *bitmap;     // rows that have an id (whole-table gradients that are overwritten), or NULL
    int32_t *lrank;       // rows form: number of the id's run in its tile
    uint32_t *hcnt;       // rows form: runs that begin in each tile
    float *part;          // [chunk][2][dim]: sums of runs that began before / go on behind the chunk
    int64_t n, bitmap_words;
    int32_t ntiles, digit;
    uint32_t none;        // key of ids without a row: the number of rows, sorted last
};

// Row and grad_out row of each id; digits of the first pass counted; the bitmap cleared.
__global__ __launch_bounds__(kSortBlock) void k_sort_start(Sort s, GradCall c) {
    __shared__ uint32_t hist[kBins];
    const int tid = threadIdx.x, bins = 1 << s.digit;
    if (s.bitmap)
        for (int64_t w = (int64_t)blockIdx.x * kSortBlock + tid; w < s.bitmap_words; w += (int64_t)gridDim.x * kSortBlock)
            s.bitmap[w] = 0;
    if ((int32_t)blockIdx.x >= s.ntiles) return;
    for (int d = tid; d < bins; d += kSortBlock) hist[d] = 0;
    __syncthreads();
    const int64_t p0 = c.offsets ? c.offsets[0] : 0, pend = c.offsets ? c.offsets[c.num_bags] : 0;
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const int64_t i = (int64_t)blockIdx.x * kSortTile + k * kSortBlock + tid;
        if (i >= s.n) break;
        const int64_t id = load_id(c.tok.ids, c.tok.index_type, i);
        const int64_t r = id == c.padding_token ? -1 : local_row(id, c.tok.first_row, c.tok.rows);
        uint32_t key = r < 0 ? s.none : (uint32_t)r;
        int64_t pay = i;
        if (c.offsets) {  // the last bag that begins at or before the id
            const int64_t p = p0 + i;
            int64_t lo = 0, hi = c.num_bags - 1;
            while (lo < hi) {
                const int64_t mid = (lo + hi + 1) >> 1;
                if (c.offsets[mid] <= p) lo = mid;
                else hi = mid - 1;
            }
            pay = lo;
            if (p >= pend) key = s.none;
        }
        s.key[0][i] = key;
        s.pay[0][i] = (int32_t)pay;
        atomicAdd(&hist[key & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int d = tid; d < bins; d += kSortBlock) s.cnt[(int64_t)blockIdx.x * bins + d] = hist[d];
}

// Digits of a later pass, tile by tile.
__global__ __launch_bounds__(kSortBlock) void k_sort_count(Sort s, int from, int shift) {
    __shared__ uint32_t hist[kBins];
    const int tid = threadIdx.x, bins = 1 << s.digit;
    for (int d = tid; d < bins; d += kSortBlock) hist[d] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const int64_t i = (int64_t)blockIdx.x * kSortTile + k * kSortBlock + tid;
        if (i < s.n) atomicAdd(&hist[(s.key[from][i] >> shift) & (bins - 1)], 1u);
    }
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
__global__ __launch_bounds__(kSortBlock) void k_sort_place(Sort s, int from, int shift, int scanned, int mark) {
    __shared__ uint32_t wcnt[kSortWaves][kBins];
    __shared__ uint32_t base[kBins];
    __shared__ int tmp[16];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bins = 1 << s.digit;
    const int32_t tile = blockIdx.x;
    for (int d = lane; d < bins; d += 64) wcnt[w][d] = 0;
    // places of the tile's first id of each digit (the scan's sums wrap only where n does: never)
    uint32_t before = 0, total = 0;
    if (tid < bins) {
        if (scanned) {
            before = s.cnt[(int64_t)tile * bins + tid];
            total = s.tot[tid];
        } else {
            for (int32_t t = 0; t < s.ntiles; ++t) {
                const uint32_t v = s.cnt[(int64_t)t * bins + tid];
                if (t < tile) before += v;
                total += v;
            }
        }
    }
    int all;
    const uint32_t smaller = (uint32_t)block_excl_scan((int)total, tmp, &all);  // its barriers order wcnt's clearing too
    if (tid < bins) base[tid] = smaller + before;
    const int64_t i0 = (int64_t)tile * kSortTile + w * kWaveKeys + lane;
    uint32_t key[kKeysPerThread], rank[kKeysPerThread];
    int32_t pay[kKeysPerThread];
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const int64_t i = i0 + k * 64;
        key[k] = i < s.n ? s.key[from][i] : 0u;
        pay[k] = i < s.n ? s.pay[from][i] : 0;
    }
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const bool valid = i0 + k * 64 < s.n;
        const uint32_t d = (key[k] >> shift) & (bins - 1);
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
        if (mark && valid && key[k] < s.none) {
            uint32_t *word = &s.bitmap[key[k] >> 5];
            const uint32_t m = 1u << (key[k] & 31);
            // repeated rows find their bit set and leave the word's queue of atomics alone
            if (!(__hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & m)) atomicOr(word, m);
        }
    }
    __syncthreads();
    if (tid < bins) {
        uint32_t run = base[tid];
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const uint32_t v = wcnt[k][tid];
            wcnt[k][tid] = run;
            run += v;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        if (i0 + k * 64 >= s.n) break;
        const uint32_t to = wcnt[w][(key[k] >> shift) & (bins - 1)] + rank[k];
        s.key[from ^ 1][to] = key[k];
        s.pay[from ^ 1][to] = pay[k];
    }
}

// Rows form: the number of each id's run in its tile (-1 before the first), runs per tile.
__global__ __launch_bounds__(kSortBlock) void k_runs(Sort s, int at) {
    __shared__ int tmp[16];
    const int64_t i0 = (int64_t)blockIdx.x * kSortTile + (int64_t)threadIdx.x * kKeysPerThread;
    const uint32_t *key = s.key[at];
    int head[kKeysPerThread], own = 0;
    uint32_t prev = i0 > 0 && i0 <= s.n ? key[i0 - 1] : s.none;
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        const uint32_t v = i0 + k < s.n ? key[i0 + k] : s.none;
        head[k] = v < s.none && (i0 + k == 0 || v != prev);
        own += head[k];
        prev = v;
    }
    int all;
    int run = block_excl_scan(own, tmp, &all) - 1;
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
        run += head[k];
        if (i0 + k < s.n) s.lrank[i0 + k] = run;
    }
    if (threadIdx.x == 0) s.hcnt[blockIdx.x] = (uint32_t)all;
}

struct SumArgs {
    int64_t nchunk;
    int32_t chunk, slices, scanned;
};

// Runs that begin before the tile of id p (rows form).  Every lane of the wave calls.
__device__ __forceinline__ int64_t runs_before(const Sort &s, int scanned, int64_t p) {
    const int32_t tile = (int32_t)(p / kSortTile);
    if (scanned) return s.hcnt[tile];
    int sum = 0;
    for (int32_t t = 0; t < tile; ++t) sum += (int)s.hcnt[t];
    return sum;
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

// Sums of one chunk's runs for one slice of LANES * V columns, per group of LANES lanes.
template <int GT, int WT, int V, int LANES>
__global__ __launch_bounds__(kSumBlock) void k_sum(Sort s, GradCall c, SumArgs a, int at) {
    constexpr int U = 4;  // rows of grad_out in flight
    const int sub = threadIdx.x & (LANES - 1);
    const uint32_t *key = s.key[at];
    const elem_t<GT> *g = static_cast<const elem_t<GT> *>(c.grad_out);
    const int64_t groups = (int64_t)gridDim.x * (kSumBlock / LANES);
    for (int64_t id = (int64_t)blockIdx.x * (kSumBlock / LANES) + threadIdx.x / LANES; id < a.nchunk * a.slices; id += groups) {
        const int64_t chunk = id / a.slices;
        const int32_t slice = (int32_t)(id - chunk * a.slices);
        const int32_t col = (slice * LANES + sub) * V, left = c.dim - col;
        const int64_t p0 = chunk * a.chunk, p1 = min(p0 + a.chunk, s.n);
        const uint32_t last = p0 > 0 ? key[p0 - 1] : s.none;
        const int64_t base = c.rows_out ? runs_before(s, a.scanned, p0) : 0;
        uint32_t cur = s.none;  // the run being summed, its row in grad, whether it began in this chunk
        int64_t row = 0;
        bool begun = true;
        float acc[V];
        int64_t done = p0;
        for (int64_t b = p0; b < p1; b += LANES) {
            const int64_t p = b + sub;
            const uint32_t kl = p < p1 ? key[p] : s.none;
            const int32_t pl = p < p1 ? s.pay[at][p] : 0;
            const unsigned long long in = __ballot(kl < s.none) >> (threadIdx.x & 63 & ~(LANES - 1));
            const int nv = __popcll(LANES == 64 ? in : in & ((1ull << LANES) - 1));  // ids without a row come last
            int32_t rl = 0;
            if (c.rows_out) {
                rl = p < p1 ? s.lrank[p] : 0;
                if (slice == 0 && sub < nv) {
                    // the lane of a run's first id names its row, that of the last id the number of rows
                    if (p == 0 || key[p - 1] != kl) c.rows_out[base + rl] = (int32_t)kl;
                    if (p + 1 == s.n || key[p + 1] == s.none) *c.count = base + rl + 1;
                }
                if (slice == 0 && p == 0 && kl == s.none) *c.count = 0;
            }
            for (int u0 = 0; u0 < nv; u0 += U) {
                float x[U][V];
                uint32_t ku[U];
                int32_t ru[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int from = min(u0 + u, nv - 1);
                    ku[u] = (uint32_t)group_read<LANES>((int)kl, from);
                    ru[u] = c.rows_out ? group_read<LANES>(rl, from) : 0;
                    const int64_t pay = group_read<LANES>(pl, from);
                    load_vec<elem_t<GT>, V>(g + pay * c.grad_out_stride + col, left, x[u]);
                }
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
                        row = c.rows_out ? base + ru[u] : (int64_t)cur;
#pragma unroll
                        for (int v = 0; v < V; ++v) acc[v] = 0.f;
                    }
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[v] += x[u][v];
                }
            }
            done = b + nv;
            if (nv < LANES) break;
        }
        if (cur == s.none) continue;
        const bool goes_on = done == p1 && p1 < s.n && key[p1] == cur;
        if (!begun) write_part<V>(s, c.dim, chunk, 0, col, left, acc);
        else if (goes_on) write_part<V>(s, c.dim, chunk, 1, col, left, acc);
        else write_row<WT, V>(c, row, col, left, acc);
    }
}

// Runs over several chunks: the block of the chunk where a run begins adds its parts.  1 << log_tc threads side by side
// on vectors of 4 columns, the others on every (1024 >> log_tc)-th part; their sums meet in LDS, in a fixed order.
template <int WT>
__global__ __launch_bounds__(kSortBlock) void k_join(Sort s, GradCall c, SumArgs a, int at, int log_tc) {
    constexpr int V = 4;
    __shared__ float red[kSortBlock * V];
    const uint32_t *key = s.key[at];
    const int tc = 1 << log_tc, groups = kSortBlock >> log_tc;
    const int x = threadIdx.x & (tc - 1), y = threadIdx.x >> log_tc;
    const int32_t col = ((int32_t)(blockIdx.y << log_tc) + x) * V, left = c.dim - col;
    for (int64_t chunk = blockIdx.x; chunk + 1 < a.nchunk; chunk += gridDim.x) {
        const int64_t p0 = chunk * a.chunk, p1 = p0 + a.chunk;
        const uint32_t k = key[p1 - 1];
        if (k == s.none || key[p1] != k || (key[p0] == k && p0 > 0 && key[p0 - 1] == k)) continue;
        int64_t end = chunk + 1;  // the last chunk whose first id belongs to the run
        for (;;) {
            const int64_t next = end + 1 + threadIdx.x;
            const int more = __syncthreads_count(next < a.nchunk && key[next * a.chunk] == k);
            end += more;
            if (more < kSortBlock) break;
        }
        float acc[V] = {0.f, 0.f, 0.f, 0.f};
        if (left > 0) {
            for (int64_t j = chunk + y; j <= end; j += groups) {
                float v[V];
                load_vec<float, V>(s.part + (j * 2 + (j == chunk ? 1 : 0)) * c.dim + col, left, v);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += v[i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) red[threadIdx.x * V + i] = acc[i];
        __syncthreads();
        if (y == 0) {
            for (int q = 1; q < groups; ++q)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += red[(q * tc + x) * V + i];
            const int64_t row = c.rows_out ? runs_before(s, a.scanned, p1 - 1) + s.lrank[p1 - 1] : (int64_t)k;
            write_row<WT, V>(c, row, col, left, acc);
        }
        __syncthreads();
    }
}

// Rows of a gradient that is overwritten and that no id names.  1 << log_tz threads side by side on a row.
template <int WT, int V>
__global__ __launch_bounds__(kSumBlock) void k_zero_rows(const uint32_t *bitmap, GradCall c, int log_tz) {
    const int tz = 1 << log_tz, ty = kSumBlock >> log_tz;
    const float zero[V] = {};
    for (int64_t r = (int64_t)blockIdx.x * ty + (threadIdx.x >> log_tz); r < c.tok.rows; r += (int64_t)gridDim.x * ty) {
        if (bitmap && (bitmap[r >> 5] >> (r & 31) & 1)) continue;
        elem_t<WT> *dst = static_cast<elem_t<WT> *>(c.grad) + r * c.grad_stride;
        for (int32_t col = (int32_t)(threadIdx.x & (tz - 1)) * V; col < c.dim; col += tz * V)
            store_vec<elem_t<WT>, V>(dst + col, c.dim - col, zero);
    }
}

__global__ void k_no_rows(int64_t *count) { *count = 0; }

int log2_ceil(int64_t x, int most) {
    int l = 0;
    while (l < most && (int64_t(1) << l) < x) ++l;
    return l;
}

unsigned capped(int64_t blocks) { return (unsigned)(blocks < 1 ? 1 : blocks > kMaxBlocks ? kMaxBlocks : blocks); }

template <int GT, int WT>
void sums_typed(const GradCall &c, const Sort &s, SumArgs a, int at, hipStream_t st) {
    constexpr int V = GT == RECMG_F32 && WT == RECMG_F32 ? 4 : 8;
    const int32_t nv = (c.dim + V - 1) / V;
    const int lanes = nv <= 16 ? 16 : nv <= 32 ? 32 : 64;
    a.slices = (nv + lanes - 1) / lanes;
    const unsigned blocks = capped((a.nchunk * a.slices * lanes + kSumBlock - 1) / kSumBlock);
    if (lanes == 16) k_sum<GT, WT, V, 16><<<blocks, kSumBlock, 0, st>>>(s, c, a, at);
    else if (lanes == 32) k_sum<GT, WT, V, 32><<<blocks, kSumBlock, 0, st>>>(s, c, a, at);
    else k_sum<GT, WT, V, 64><<<blocks, kSumBlock, 0, st>>>(s, c, a, at);
    if (a.nchunk > 1) {
        const int log_tc = log2_ceil((c.dim + 3) / 4, 8);
        const dim3 grid(capped(a.nchunk - 1), (unsigned)((c.dim + (4 << log_tc) - 1) / (4 << log_tc)));
        k_join<WT><<<grid, kSortBlock, 0, st>>>(s, c, a, at, log_tc);
    }
}

template <int WT>
void zero_typed(const GradCall &c, const uint32_t *bitmap, hipStream_t st) {
    constexpr int V = WT == RECMG_F32 ? 4 : 8;
    const int log_tz = log2_ceil((c.dim + V - 1) / V, 8);
    k_zero_rows<WT, V><<<capped((c.tok.rows << log_tz) / kSumBlock + 1), kSumBlock, 0, st>>>(bitmap, c, log_tz);
}

size_t take(size_t *at, size_t bytes) {
    const size_t here = *at;
    *at += (bytes + 255) & ~size_t(255);
    return here;
}

}  // namespace

GradPlan grad_plan(int64_t rows, int32_t dim, int64_t n, bool rows_form) {
    GradPlan p{};
    if (n == 0) return p;
    p.ntiles = (int32_t)((n + kSortTile - 1) / kSortTile);
    int bits = 1;
    while (rows >> bits) ++bits;  // the key of ids without a row is `rows` itself
    p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    p.digit = (bits + p.passes - 1) / p.passes;
    // chunks: short ones while there are few ids (some 8,192 waves fill the chip), long ones, whose ends cost less, beyond
    const int64_t waves = n * ((dim + 511) / 512);
    p.chunk = 16;
    while (p.chunk < 512 && waves / p.chunk > 8192) p.chunk *= 2;
    p.nchunk = (n + p.chunk - 1) / p.chunk;
    p.bitmap_words = rows_form ? 0 : (rows + 31) / 32;
    for (int k = 0; k < 2; ++k) {
        p.key[k] = take(&p.total, n * 4);
        p.pay[k] = take(&p.total, n * 4);
    }
    p.cnt = take(&p.total, ((size_t)p.ntiles << p.digit) * 4);
    p.tot = take(&p.total, (size_t)kBins * 4);
    p.bitmap = take(&p.total, p.bitmap_words * 4);
    p.lrank = take(&p.total, rows_form ? n * 4 : 0);
    p.hcnt = take(&p.total, rows_form ? (size_t)p.ntiles * 4 : 0);
    p.part = take(&p.total, (size_t)p.nchunk * 2 * dim * 4);
    return p;
}

void launch_row_gradient(const GradCall &c, const GradPlan &p, char *ws, hipStream_t st) {
    const bool rows_form = c.rows_out != nullptr;
    const bool fill = !rows_form && !c.accumulate;
    Sort s{};
    if (c.tok.n > 0) {
        for (int k = 0; k < 2; ++k) {
            s.key[k] = reinterpret_cast<uint32_t *>(ws + p.key[k]);
            s.pay[k] = reinterpret_cast<int32_t *>(ws + p.pay[k]);
        }
        s.cnt = reinterpret_cast<uint32_t *>(ws + p.cnt);
        s.tot = reinterpret_cast<uint32_t *>(ws + p.tot);
        s.bitmap = fill ? reinterpret_cast<uint32_t *>(ws + p.bitmap) : nullptr;
        s.lrank = reinterpret_cast<int32_t *>(ws + p.lrank);
        s.hcnt = reinterpret_cast<uint32_t *>(ws + p.hcnt);
        s.part = reinterpret_cast<float *>(ws + p.part);
        s.n = c.tok.n;
        s.bitmap_words = fill ? p.bitmap_words : 0;
        s.ntiles = p.ntiles;
        s.digit = p.digit;
        s.none = (uint32_t)c.tok.rows;
        const int scanned = p.ntiles > kScanTiles;
        const int bins = 1 << p.digit;
        // more blocks than tiles only clear the bitmap
        const int64_t clear = (s.bitmap_words + 16 * kSortBlock - 1) / (16 * kSortBlock);
        k_sort_start<<<(unsigned)(clear > p.ntiles ? clear : p.ntiles), kSortBlock, 0, st>>>(s, c);
        for (int q = 0; q < p.passes; ++q) {
            if (q > 0) k_sort_count<<<p.ntiles, kSortBlock, 0, st>>>(s, q & 1, q * p.digit);
            if (scanned) k_scan_tiles<<<(bins + 63) / 64, kSortBlock, 0, st>>>(s.cnt, s.tot, p.ntiles, bins);
            k_sort_place<<<p.ntiles, kSortBlock, 0, st>>>(s, q & 1, q * p.digit, scanned, fill && q == 0);
        }
        const int at = p.passes & 1;
        if (rows_form) {
            k_runs<<<p.ntiles, kSortBlock, 0, st>>>(s, at);
            if (scanned) k_scan_tiles<<<1, kSortBlock, 0, st>>>(s.hcnt, s.tot, p.ntiles, 1);
        }
        const SumArgs a{p.nchunk, p.chunk, 0, scanned};
#define RECMG_CASE(A, B) \
    case A * 3 + B: sums_typed<A, B>(c, s, a, at, st); break;
        switch (c.grad_out_dtype * 3 + c.grad_dtype) {
            RECMG_CASE(0, 0) RECMG_CASE(0, 1) RECMG_CASE(0, 2)
            RECMG_CASE(1, 0) RECMG_CASE(1, 1) RECMG_CASE(1, 2)
            RECMG_CASE(2, 0) RECMG_CASE(2, 1) RECMG_CASE(2, 2)
        }
#undef RECMG_CASE
    } else if (rows_form) {
        k_no_rows<<<1, 1, 0, st>>>(c.count);
    }
    if (fill) {
        if (c.grad_dtype == RECMG_F32) zero_typed<RECMG_F32>(c, s.bitmap, st);
        else if (c.grad_dtype == RECMG_F16) zero_typed<RECMG_F16>(c, s.bitmap, st);
        else zero_typed<RECMG_BF16>(c, s.bitmap, st);
    }
}

}  // namespace recmg
