// The norm of many gradients, sqrt(sum of g^2), and their clipping,
// out = g * min(1, max_norm / (norm + eps)).
//
// Each is one pass over the tensors, bound by HBM.  A launch takes the tensors
// as one sequence of chunks of up to 16,384 elements, so short tensors cost what their
// elements cost and long ones spread over all blocks.
//
// Squares and sums are in 64 bits: a square of an fp32 or bf16 value leaves the
// fp32 range from about 1e19 up and 1e-19 down, and the vector units add and
// multiply doubles faster than HBM brings values.  Every block writes one sum and
// one block adds them, in a fixed order: the norm is the same from call to call.
#include <float.h>

#include "gradients.h"
#include "values.h"

namespace recmg {

namespace {

constexpr int kGradBlock = 256;

// The tensor that chunk c belongs to.
__device__ __forceinline__ int tensor_of(const GradTensors &t, int64_t c) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// The elements [e0, e1) of tensor k that chunk c holds, without the rows behind a count.
__device__ __forceinline__ void chunk_elements(const GradTensors &t, int k, int64_t c, int64_t *e0, int64_t *e1) {
    *e0 = (c - t.first[k]) * t.chunk;
    *e1 = c + 1 == t.first[k + 1] ? *e0 + t.tail[k] + 1 : *e0 + t.chunk;
    for (int q = 0; q < t.live; ++q)
        if (t.live_of[q] == k) {
            const int64_t rows = *t.live_rows[q], len = t.live_len[q];
            const int64_t n = rows <= 0 ? 0 : rows > kMostElements / len ? kMostElements : rows * len;
            if (*e1 > n) *e1 = n > *e0 ? n : *e0;
        }
}

// U vectors of V elements from p on, a block's width apart; `left` elements from p on, all of them if `whole` (the same in
// all lanes: no branches between the loads then).  What lies behind is 0.
template <typename T, int V, int U>
__device__ __forceinline__ void load_strip(const T *p, int64_t left, bool whole, float (&x)[U][V]) {
    if (whole) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_whole<T, V>(p + u * kGradBlock * V, x[u]);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t l = left - u * kGradBlock * V;
            load_vec<T, V>(p + u * kGradBlock * V, (int32_t)(l < 0 ? 0 : l), x[u]);
        }
    }
}

// Sum of the squares of the elements [e0, e1) that this thread takes.
template <int DT>
__device__ __forceinline__ double squares(const void *src, int64_t e0, int64_t e1) {
    constexpr int V = DT == RECMG_F32 ? 4 : 8;
    constexpr int U = 2;  // vectors in flight (1, 2, 4, 8: 148, 150, 161, 158 us for 800 MB of 290 tensors)
    const elem_t<DT> *p = static_cast<const elem_t<DT> *>(src);
    constexpr int64_t kStrip = (int64_t)U * kGradBlock * V;
    double sum[2] = {0.0, 0.0};
    for (int64_t e = e0; e < e1; e += kStrip) {
        float x[U][V];
        const int64_t at = e + (int64_t)threadIdx.x * V;
        load_strip<elem_t<DT>, V, U>(p + at, e1 - at, e + kStrip <= e1, x);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v & 1] = __builtin_fma((double)x[u][v], (double)x[u][v], sum[v & 1]);
    }
    return sum[0] + sum[1];
}

// Sum over the block's threads, in thread 0.
__device__ __forceinline__ double block_sum_f64(double v) {
    __shared__ double tmp[kGradBlock / 64];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int k = 0; k < kGradBlock / 64; ++k) s += tmp[k];
    return s;
}

// Blocks side by side take chunks side by side (800 MB of 290 tensors: 152 us; each a range of its own: 160).
__global__ __launch_bounds__(kGradBlock) void k_norm_sums(GradTensors t, double *partial) {
    double sum = 0.0;
    for (int64_t c = blockIdx.x; c < t.first[t.count]; c += gridDim.x) {
        const int k = tensor_of(t, c);
        int64_t e0, e1;
        chunk_elements(t, k, c, &e0, &e1);
        switch (t.types[k] & 3) {
            case RECMG_F32: sum += squares<RECMG_F32>(t.src[k], e0, e1); break;
            case RECMG_F16: sum += squares<RECMG_F16>(t.src[k], e0, e1); break;
            default: sum += squares<RECMG_BF16>(t.src[k], e0, e1);
        }
    }
    sum = block_sum_f64(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// The norm, in every thread, from the partial sums: the same order in every block.
__device__ __forceinline__ double norm_of(const double *partial, int64_t sums) {
    __shared__ double norm;
    double v = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < sums; i += kGradBlock) v += partial[i];
    v = block_sum_f64(v);
    if (threadIdx.x == 0) norm = __builtin_sqrt(v);
    __syncthreads();
    return norm;
}

// The norm to *norm, and in 64 bits to partial[0], where clipping reads it (the partial sums have been read by then).
__global__ __launch_bounds__(kGradBlock) void k_norm_end(double *partial, int64_t sums, float *norm) {
    const double v = norm_of(partial, sums);
    if (threadIdx.x == 0) {
        *norm = (float)v;
        partial[0] = v;
    }
}

// mant * 2^exp.  exp = 0, but where fp32 holds the factor with fewer bits than a normal number has: 1e37 * (1e-3 / 1e38) is
// 1e-4, far from fp32's end.  (Products in 64 bits for such factors would cost every call: 12.7 -> 16.3 us for 62 tensors of 2
// million elements, of the kernel's size and registers alone.)
struct Factor {
    float mant;
    int exp;
};

template <int ST, int DT>
__device__ __forceinline__ void scale_chunk(const void *src, void *dst, int64_t e0, int64_t e1, const Factor &c) {
    constexpr int V = ST == RECMG_F32 && DT == RECMG_F32 ? 4 : 8;
    constexpr int U = 8;  // vectors in flight (1, 2, 4, 8: 511, 493, 486, 469 us, the norm before it too, for 600 MB to 1.2 GB)
    const elem_t<ST> *p = static_cast<const elem_t<ST> *>(src);
    elem_t<DT> *q = static_cast<elem_t<DT> *>(dst);
    constexpr int64_t kStrip = (int64_t)U * kGradBlock * V;
    for (int64_t e = e0; e < e1; e += kStrip) {
        float x[U][V];
        const int64_t at = e + (int64_t)threadIdx.x * V;
        load_strip<elem_t<ST>, V, U>(p + at, e1 - at, e + kStrip <= e1, x);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t left = e1 - at - u * kGradBlock * V;
#pragma unroll
            for (int v = 0; v < V; ++v) x[u][v] = __builtin_ldexpf(x[u][v] * c.mant, c.exp);
            if (left > 0) store_vec<elem_t<DT>, V>(q + at + u * kGradBlock * V, (int32_t)left, x[u]);
        }
    }
}

// FUSED: the norm from partial sums, which block 0 writes too; else it is read, in 64 bits where k_norm_end has left it.
template <bool FUSED>
__global__ __launch_bounds__(kGradBlock) void k_clip(GradTensors t, const double *partial, int64_t sums, float *norm,
                                                     float max_norm, float eps) {
    double length;
    if constexpr (FUSED) {
        length = norm_of(partial, sums);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)length;
    } else {
        length = partial ? partial[0] : (double)*norm;
    }
    // a norm that is no number makes the factor and every value none; an infinite one makes it 0, whatever the limit
    double f = __builtin_isinf(length) ? 0.0 : (double)max_norm / (length + (double)eps);
    if (f > 1.0) f = 1.0;
    Factor factor{(float)f, 0};
    if (f < (double)FLT_MIN) factor.mant = (float)__builtin_frexp(f, &factor.exp);
    const bool all = factor.mant == 1.f && factor.exp == 0;
    if (all && t.in_place) return;  // nothing changes
    for (int64_t c = blockIdx.x; c < t.first[t.count]; c += gridDim.x) {
        const int k = tensor_of(t, c);
        if (all && t.src[k] == t.dst[k]) continue;
        int64_t e0, e1;
        chunk_elements(t, k, c, &e0, &e1);
        switch (t.types[k]) {
#define RECMG_CASE(A, B) \
    case A + 4 * B: scale_chunk<A, B>(t.src[k], t.dst[k], e0, e1, factor); break;
            RECMG_CASE(0, 0) RECMG_CASE(0, 1) RECMG_CASE(0, 2)
            RECMG_CASE(1, 0) RECMG_CASE(1, 1) RECMG_CASE(1, 2)
            RECMG_CASE(2, 0) RECMG_CASE(2, 1) RECMG_CASE(2, 2)
#undef RECMG_CASE
        }
    }
}

}  // namespace

int launch_norm_sums(const GradTensors &t, double *partial, int most, Launches &run) {
    const int blocks = t.first[t.count] < most ? t.first[t.count] : most;
    run(k_norm_sums, blocks, kGradBlock, t, partial);
    return blocks;
}

void launch_norm_end(double *partial, int64_t sums, float *norm, Launches &run) {
    run(k_norm_end, 1, kGradBlock, partial, sums, norm);
}

void launch_clip(const GradTensors &t, const double *partial, int64_t sums, float *norm, float max_norm, float eps,
                 Launches &run) {
    // a block per chunk, where the chunks have to be written; gradients in place mostly stay within the limit, and few
    // blocks then find that out sooner
    const int64_t chunks = t.first[t.count], most = t.in_place ? 8192 : 1 << 20;
    const unsigned blocks = (unsigned)(chunks < most ? chunks : most);
    if (sums > 0) run(k_clip<true>, blocks, kGradBlock, t, partial, sums, norm, max_norm, eps);
    else run(k_clip<false>, blocks, kGradBlock, t, partial, sums, norm, max_norm, eps);
}

}  // namespace recmg
