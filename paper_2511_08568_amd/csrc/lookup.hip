// Token lookup: out[i, :] = round(scale * table[tokens[i] - first_row, :]), rows
// of zeros for tokens whose row the table does not hold.
//
// It reads each distinct row once at least and writes every output row once: the
// writes are most of it, and HBM bounds it; a few tokens are bound by the chain
// token id -> row -> store and the launch.
#include "embedding.h"
#include "values.h"

namespace recmg {

namespace {

constexpr int kLookupLog = 9, kLookupBlock = 1 << kLookupLog;
constexpr int64_t kMaxBlocks = 1 << 20;  // a launch holds fewer than 2^32 threads; blocks take several shares beyond
// Outputs above this bypass the caches: they would push the table's rows out, and the caches (256 MiB in all) could
// not keep them for the next kernel.  131,072 x 4,096 bf16: 269 us against 285.  Smaller ones gain as much (8,192 x
// 2,048: 10.2 us against 11.4) as the kernel that reads them next loses.
constexpr int64_t kStreamBytes = 128 << 20;

// A thread takes one vector of V columns of R rows: the R token ids, then the R
// row pieces are in flight together (R = 1, 2, 4, 8: 323, 269, 320, 354 us for
// 131,072 x 4,096 bf16).  tx threads (a power of two) side by side on a row, a
// whole row of up to 8 KiB where there are so many; blockIdx.y counts pieces of
// tx vectors.
template <int TT, int TO, int V, int R>
__global__ __launch_bounds__(kLookupBlock) void k_lookup(const elem_t<TT> *__restrict__ table, int64_t table_stride,
                                                         Tokens tok, int32_t dim, int log_tx, float scale,
                                                         elem_t<TO> *__restrict__ out, int64_t out_stride, int stream_out) {
    const int tx = 1 << log_tx, ty = kLookupBlock >> log_tx;
    const int32_t col = ((int32_t)(blockIdx.y << log_tx) + (int32_t)(threadIdx.x & (tx - 1))) * V;
    const int32_t left = dim - col;
    if (left <= 0) return;
    for (int64_t i0 = (int64_t)blockIdx.x * (ty * R) + (threadIdx.x >> log_tx); i0 < tok.n;
         i0 += (int64_t)gridDim.x * (ty * R)) {
        int64_t row[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t i = i0 + k * ty;  // behind the last: as the last, and not stored
            row[k] = local_row(load_id(tok.ids, tok.index_type, i < tok.n ? i : tok.n - 1), tok.first_row, tok.rows);
        }
        float x[R][V];
        // tokens without a row read row 0
        load_vecs<elem_t<TT>, V, R>(dim % V == 0, left, [&](int k) { return table + (row[k] >= 0 ? row[k] : 0) * table_stride + col; }, x);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t i = i0 + k * ty;
            if (i >= tok.n) break;
#pragma unroll
            for (int v = 0; v < V; ++v) x[k][v] = row[k] >= 0 ? x[k][v] * scale : 0.f;
            if (stream_out) store_vec<elem_t<TO>, V, STREAM>(out + i * out_stride + col, left, x[k]);
            else store_vec<elem_t<TO>, V>(out + i * out_stride + col, left, x[k]);
        }
    }
}

template <int TT, int TO>
void lookup_typed(const void *table, int64_t table_stride, const Tokens &tok, int32_t dim, float scale, void *out,
                  int64_t out_stride, Launches &run) {
    constexpr int V = TT == RECMG_F32 && TO == RECMG_F32 ? 4 : 8;  // 16 bytes of the narrower type
    const int32_t nv = (dim + V - 1) / V;
    int log_tx = 0;
    while ((1 << log_tx) < nv && log_tx < kLookupLog) ++log_tx;
    const int ty = kLookupBlock >> log_tx;
    constexpr int R = 2;
    const int64_t blocks = (tok.n + ty * R - 1) / (ty * R);
    const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks), (unsigned)((nv + (1 << log_tx) - 1) >> log_tx));
    const elem_t<TT> *t = static_cast<const elem_t<TT> *>(table);
    elem_t<TO> *o = static_cast<elem_t<TO> *>(out);
    const int stream_out = tok.n * dim * (int64_t)sizeof(elem_t<TO>) > kStreamBytes;
    run(k_lookup<TT, TO, V, R>, grid, kLookupBlock, t, table_stride, tok, dim, log_tx, scale, o, out_stride, stream_out);
}

}  // namespace

void launch_lookup(const void *table, int32_t table_dtype, int64_t table_stride, const Tokens &tok, int32_t dim,
                   float scale, void *out, int32_t out_dtype, int64_t out_stride, Launches &run) {
#define RECMG_CASE(A, B) \
    case A * 3 + B: return lookup_typed<A, B>(table, table_stride, tok, dim, scale, out, out_stride, run);
    switch (table_dtype * 3 + out_dtype) {
        RECMG_CASE(0, 0) RECMG_CASE(0, 1) RECMG_CASE(0, 2)
        RECMG_CASE(1, 0) RECMG_CASE(1, 1) RECMG_CASE(1, 2)
        RECMG_CASE(2, 0) RECMG_CASE(2, 1) RECMG_CASE(2, 2)
    }
#undef RECMG_CASE
}

}  // namespace recmg
