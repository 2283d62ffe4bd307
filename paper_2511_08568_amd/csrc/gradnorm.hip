// The norm of many gradients, sqrt(sum of g^2), and their clipping,
// out = g * min(1, max_norm / (norm + eps)).
//
// Each is one pass over the tensors, bound by HBM.  A launch takes the tensors
// as one sequence of chunks of 16,384 elements, so short tensors cost what their
// elements cost and long ones spread over all blocks.
//
// Squares and sums are in 64 bits: a square of an fp32 or bf16 value leaves the
// fp32 range from about 1e19 up and 1e-19 down, and the vector units add and
// multiply doubles faster than HBM brings values.  Every block writes one sum and
// one block adds them, in a fixed order: the norm is the same from call to call.
#include "gradients.h"
#include "values.h"

namespace recmg {

namespace {

constexpr int kGradBlock = 256;

// Elements of tensor k that hold values.
__device__ __forceinline__ int64_t live_elements(const GradTensors &t, int k) {
    const int64_t n = t.numel[k];
    if (!t.live[k]) return n;
    const int64_t rows = *t.live[k];
    const int64_t len = t.row_len[k];
    return rows <= 0 ? 0 : rows >= (n + len - 1) / len ? n : rows * len;
}

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

// Sum of the squares of the elements [e0, e1) that this thread takes.
template <int DT>
__device__ __forceinline__ double squares(const void *src, int64_t e0, int64_t e1) {
    constexpr int V = DT == RECMG_F32 ? 4 : 8;
    constexpr int U = 4;  // vectors in flight
    const elem_t<DT> *p = static_cast<const elem_t<DT> *>(src);
    double sum[2] = {0.0, 0.0};
    for (int64_t e = e0 + (int64_t)threadIdx.x * V; e < e1; e += (int64_t)U * kGradBlock * V) {
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = e + (int64_t)u * kGradBlock * V;
            load_vec<elem_t<DT>, V>(p + at, (int32_t)(e1 - at < 0 ? 0 : e1 - at), x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v & 1] = __builtin_fma((double)x[u][v], (double)x[u][v], sum[v & 1]);
    }
    return sum[0] + sum[1];
}

// Sum over the block's threads, in thread 0.
template <int BLOCK>
__device__ __forceinline__ double block_sum_f64(double v) {
    __shared__ double tmp[BLOCK / 64];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int k = 0; k < BLOCK / 64; ++k) s += tmp[k];
    return s;
}

__global__ __launch_bounds__(kGradBlock) void k_norm_sums(GradTensors t, double *partial) {
    const int64_t c0 = t.chunks * blockIdx.x / gridDim.x, c1 = t.chunks * (blockIdx.x + 1) / gridDim.x;
    double sum = 0.0;
    int k = tensor_of(t, c0);
    for (int64_t c = c0; c < c1; ++c) {
        while (k + 1 < t.count && t.first[k + 1] <= c) ++k;
        const int64_t e0 = (c - t.first[k]) * kGradChunk, n = live_elements(t, k);
        const int64_t e1 = e0 + kGradChunk < n ? e0 + kGradChunk : n;
        switch (t.types[k] & 3) {
            case RECMG_F32: sum += squares<RECMG_F32>(t.src[k], e0, e1); break;
            case RECMG_F16: sum += squares<RECMG_F16>(t.src[k], e0, e1); break;
            default: sum += squares<RECMG_BF16>(t.src[k], e0, e1);
        }
    }
    sum = block_sum_f64<kGradBlock>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void k_norm_end(const double *partial, int64_t sums, float *norm) {
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < sums; i += 1024) v += partial[i];
    v = block_sum_f64<1024>(v);
    if (threadIdx.x == 0) *norm = (float)__builtin_sqrt(v);
}

template <int ST, int DT>
__device__ __forceinline__ void scale_chunk(const void *src, void *dst, int64_t e0, int64_t e1, float c) {
    constexpr int V = ST == RECMG_F32 && DT == RECMG_F32 ? 4 : 8;
    constexpr int U = 4;
    const elem_t<ST> *p = static_cast<const elem_t<ST> *>(src);
    elem_t<DT> *q = static_cast<elem_t<DT> *>(dst);
    for (int64_t e = e0 + (int64_t)threadIdx.x * V; e < e1; e += (int64_t)U * kGradBlock * V) {
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = e + (int64_t)u * kGradBlock * V;
            load_vec<elem_t<ST>, V>(p + at, (int32_t)(e1 - at < 0 ? 0 : e1 - at), x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = e + (int64_t)u * kGradBlock * V;
#pragma unroll
            for (int v = 0; v < V; ++v) x[u][v] *= c;
            if (at < e1) store_vec<elem_t<DT>, V>(q + at, (int32_t)(e1 - at), x[u]);
        }
    }
}

__global__ __launch_bounds__(kGradBlock) void k_clip(GradTensors t, const float *norm, float max_norm, float eps) {
    // a norm that is no number makes the factor and every value none; an infinite one makes it 0
    float f = (float)((double)max_norm / ((double)*norm + (double)eps));
    if (f > 1.f) f = 1.f;
    for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int k = tensor_of(t, c);
        if (f == 1.f && t.src[k] == t.dst[k]) continue;  // in place: nothing changes
        const int64_t e0 = (c - t.first[k]) * kGradChunk, n = live_elements(t, k);
        const int64_t e1 = e0 + kGradChunk < n ? e0 + kGradChunk : n;
        switch (t.types[k]) {
#define RECMG_CASE(A, B) \
    case A + 4 * B: scale_chunk<A, B>(t.src[k], t.dst[k], e0, e1, f); break;
            RECMG_CASE(0, 0) RECMG_CASE(0, 1) RECMG_CASE(0, 2)
            RECMG_CASE(1, 0) RECMG_CASE(1, 1) RECMG_CASE(1, 2)
            RECMG_CASE(2, 0) RECMG_CASE(2, 1) RECMG_CASE(2, 2)
#undef RECMG_CASE
        }
    }
}

}  // namespace

int launch_norm_sums(const GradTensors &t, double *partial, hipStream_t s) {
    const int blocks = (int)(t.chunks < kNormBlocks ? t.chunks : kNormBlocks);
    k_norm_sums<<<blocks, kGradBlock, 0, s>>>(t, partial);
    return blocks;
}

void launch_norm_end(const double *partial, int64_t sums, float *norm, hipStream_t s) {
    k_norm_end<<<1, 1024, 0, s>>>(partial, sums, norm);
}

void launch_clip(const GradTensors &t, const float *norm, float max_norm, float eps, hipStream_t s) {
    const int64_t blocks = t.chunks < (1 << 20) ? t.chunks : 1 << 20;
    k_clip<<<(unsigned)blocks, kGradBlock, 0, s>>>(t, norm, max_norm, eps);
}

}  // namespace recmg
