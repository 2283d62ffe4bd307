// C entries of the token-embedding lookup and its gradient: checks of the
// arguments, the workspace's layout, the launches.
#include "embedding.h"
#include "status.h"
#include "values.h"

using namespace recmg;

namespace {

bool bad_dtype(int32_t d) { return d != RECMG_F32 && d != RECMG_F16 && d != RECMG_BF16; }

// RECMG_OK, or the refusal of a matrix of `count` rows (its name in the message).
int32_t check_matrix(const char *name, const void *data, int32_t dtype, int64_t stride, int64_t least, int32_t dim,
                     int64_t count) {
    if (bad_dtype(dtype)) return fail(RECMG_E_INVALID, std::string("bad dtype of ") + name);
    if (stride < least || stride > (int64_t(1) << 40))
        return fail(RECMG_E_INVALID, std::string("row stride out of range: ") + name);
    if (count > 0 && !data) return fail(RECMG_E_INVALID, std::string(name) + " is NULL");
    if (reinterpret_cast<uintptr_t>(data) % elem_size(dtype))
        return fail(RECMG_E_INVALID, std::string(name) + " is not aligned to its elements");
    return RECMG_OK;
}

int32_t check_tokens(const Tokens &t, int32_t dim) {
    if (t.rows < 1 || t.rows >= (int64_t(1) << 31)) return fail(RECMG_E_INVALID, "rows out of [1, 2^31)");
    if (dim < 1 || dim > (1 << 16)) return fail(RECMG_E_INVALID, "dim out of [1, 65536]");
    if (t.index_type != RECMG_I32 && t.index_type != RECMG_I64) return fail(RECMG_E_INVALID, "bad index_type");
    if (t.n < 0 || t.n >= (int64_t(1) << 31)) return fail(RECMG_E_INVALID, "num_tokens out of [0, 2^31)");
    if (t.first_row < 0) return fail(RECMG_E_INVALID, "negative first_row");
    if (t.n > 0 && !t.ids) return fail(RECMG_E_INVALID, "tokens is NULL");
    if (reinterpret_cast<uintptr_t>(t.ids) % (t.index_type == RECMG_I32 ? 4 : 8))
        return fail(RECMG_E_INVALID, "tokens is not aligned to its elements");
    return RECMG_OK;
}

// Bytes that a call reads or writes: n rows of `width`, `stride` from one to the next.
struct Bytes {
    const char *name;
    __int128 at;
    __int128 stride, n, width;
};

Bytes bytes_of(const char *name, const void *p, int64_t n, int64_t width, int64_t stride) {
    Bytes b{name, (__int128)reinterpret_cast<uintptr_t>(p), stride, n, width};
    if (n > 0 && stride <= width) {  // one range without gaps (a stride of 0: one row)
        b.width += (b.n - 1) * b.stride;
        b.n = 1;
    }
    return b;
}

// Whether two of them share a byte; false also for row strides that differ where neither is one range.
bool share(const Bytes &a, const Bytes &b) {
    if (a.n < 1 || b.n < 1) return false;
    if (a.at + (a.n - 1) * a.stride + a.width <= b.at || b.at + (b.n - 1) * b.stride + b.width <= a.at) return false;
    if (a.n == 1 && b.n == 1) return true;
    if (a.n == 1) return share(b, a);
    const auto down = [&](__int128 x) { return x >= 0 ? x / a.stride : -((-x + a.stride - 1) / a.stride); };
    if (b.n == 1) {  // the first row of a that ends behind b's begin
        const __int128 i = down(b.at - a.width - a.at) + 1, row = i < 0 ? 0 : i;
        return row < a.n && a.at + row * a.stride < b.at + b.width;
    }
    if (a.stride != b.stride) return false;
    // row j of b begins d + (j - i) * stride behind row i of a: they share bytes where that is in (-b.width, a.width)
    const __int128 d = b.at - a.at, m = -down(d), q = d + m * a.stride;  // 0 <= q < stride
    const auto rows = [&](__int128 k) { return k >= 1 - a.n && k <= b.n - 1; };  // some i and j with j - i = k
    return (q < a.width && rows(m)) || (q - a.stride > -b.width && rows(m - 1));
}

// Refuses outputs that share memory with what the call reads, or with one another.
int32_t check_apart(const Bytes *outs, int n_outs, const Bytes *ins, int n_ins) {
    for (int o = 0; o < n_outs; ++o) {
        for (int k = 0; k < n_ins + o; ++k) {
            const Bytes &other = k < n_ins ? ins[k] : outs[k - n_ins];
            if (share(outs[o], other)) return fail(RECMG_E_INVALID, std::string(outs[o].name) + " shares memory with " + other.name);
        }
    }
    return RECMG_OK;
}

Bytes matrix_bytes(const char *name, const void *p, int32_t dtype, int64_t stride, int32_t dim, int64_t n) {
    const int64_t size = elem_size(dtype);
    return bytes_of(name, p, n, dim * size, stride * size);
}

Bytes token_bytes(const Tokens &t) { return bytes_of("tokens", t.ids, t.n > 0 ? 1 : 0, t.n * (t.index_type == RECMG_I32 ? 4 : 8), 0); }

// What both forms of the gradient take and check alike.
int32_t check_gradient(const GradCall &c) {
    int32_t rc = check_tokens(c.tok, c.dim);
    if (rc) return rc;
    if (c.offsets) {
        if (c.num_bags < 0 || c.num_bags >= (int64_t(1) << 31)) return fail(RECMG_E_INVALID, "num_bags out of [0, 2^31)");
        if (reinterpret_cast<uintptr_t>(c.offsets) % 8) return fail(RECMG_E_INVALID, "offsets is not aligned to 8 bytes");
    }
    // one row of grad_out may stand for all (stride 0), as where a sum's gradient is expanded
    if ((rc = check_matrix("grad_out", c.grad_out, c.grad_out_dtype, c.grad_out_stride, 0, c.dim,
                           c.offsets ? c.num_bags : c.tok.n)))
        return rc;
    return RECMG_OK;
}

int32_t run_gradient(const GradCall &c, void *workspace, size_t workspace_bytes, void *stream) {
    const GradPlan p = grad_plan(c.tok.rows, c.dim, c.tok.n, c.rows_out != nullptr, c.offsets != nullptr);
    if (p.total > 0) {
        if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256)
            return fail(RECMG_E_INVALID, "workspace is NULL or not aligned to 256 bytes");
        if (workspace_bytes < p.total)
            return fail(RECMG_E_NOMEM, "workspace smaller than recmg_query_embedding_workspace says");
    }
    const bool rows_form = c.rows_out != nullptr;
    const int64_t most = c.tok.n < c.tok.rows ? c.tok.n : c.tok.rows;
    const Bytes ins[] = {matrix_bytes("grad_out", c.grad_out, c.grad_out_dtype, c.grad_out_stride, c.dim, c.offsets ? c.num_bags : c.tok.n),
                         token_bytes(c.tok), bytes_of("offsets", c.offsets, c.offsets ? 1 : 0, (c.num_bags + 1) * 8, 0)};
    const Bytes outs[] = {matrix_bytes(rows_form ? "values" : "grad", c.grad, c.grad_dtype, c.grad_stride, c.dim, rows_form ? most : c.tok.rows),
                          bytes_of("workspace", workspace, p.total > 0 ? 1 : 0, (int64_t)p.total, 0),
                          bytes_of("rows_out", c.rows_out, rows_form && most > 0 ? 1 : 0, most * 4, 0),
                          bytes_of("count", c.count, rows_form ? 1 : 0, 8, 0)};
    if (const int32_t rc = check_apart(outs, 4, ins, 3)) return rc;
    Launches run{static_cast<hipStream_t>(stream)};
    launch_row_gradient(c, p, static_cast<char *>(workspace), run);
    return run.status();
}

}  // namespace

extern "C" {

int32_t recmg_embedding_forward(const void *table, int32_t table_dtype, int64_t table_stride, int64_t rows, int32_t dim,
                                const void *tokens, int32_t index_type, int64_t num_tokens, int64_t first_row,
                                float scale, void *out, int32_t out_dtype, int64_t out_stride, void *stream) {
    const Tokens tok{tokens, num_tokens, first_row, rows, index_type};
    int32_t rc = check_tokens(tok, dim);
    if (rc) return rc;
    if ((rc = check_matrix("table", table, table_dtype, table_stride, dim, dim, rows))) return rc;
    if ((rc = check_matrix("out", out, out_dtype, out_stride, dim, dim, num_tokens))) return rc;
    if (num_tokens == 0) return RECMG_OK;
    const Bytes ins[] = {matrix_bytes("table", table, table_dtype, table_stride, dim, rows), token_bytes(tok)};
    const Bytes o = matrix_bytes("out", out, out_dtype, out_stride, dim, num_tokens);
    if ((rc = check_apart(&o, 1, ins, 2))) return rc;
    Launches run{static_cast<hipStream_t>(stream)};
    launch_lookup(table, table_dtype, table_stride, tok, dim, scale, out, out_dtype, out_stride, run);
    return run.status();
}

int32_t recmg_query_embedding_workspace(int64_t rows, int32_t dim, int64_t num_tokens, int32_t rows_form, int32_t bags,
                                        size_t *bytes) {
    if (!bytes) return fail(RECMG_E_INVALID, "bytes is NULL");
    static const int64_t aligned = 0;  // any address: only the sizes are checked here
    const int32_t rc = check_tokens(Tokens{&aligned, num_tokens, 0, rows, RECMG_I32}, dim);
    if (rc) return rc;
    *bytes = grad_plan(rows, dim, num_tokens, rows_form != 0, bags != 0).total;
    return RECMG_OK;
}

int32_t recmg_embedding_backward(const void *grad_out, int32_t grad_out_dtype, int64_t grad_out_stride, const void *tokens,
                                 int32_t index_type, int64_t num_tokens, const int64_t *offsets, int64_t num_bags,
                                 int64_t rows, int32_t dim, int64_t first_row, int64_t padding_token, float scale,
                                 void *grad, int32_t grad_dtype, int64_t grad_stride, int32_t accumulate,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    const GradCall c{Tokens{tokens, num_tokens, first_row, rows, index_type}, padding_token, offsets, num_bags, dim, scale,
                     grad_out, grad_out_dtype, grad_out_stride, grad, grad_dtype, grad_stride, accumulate != 0,
                     nullptr, nullptr};
    int32_t rc = check_gradient(c);
    if (rc) return rc;
    if ((rc = check_matrix("grad", grad, grad_dtype, grad_stride, dim, dim, rows))) return rc;
    return run_gradient(c, workspace, workspace_bytes, stream);
}

int32_t recmg_embedding_backward_rows(const void *grad_out, int32_t grad_out_dtype, int64_t grad_out_stride,
                                      const void *tokens, int32_t index_type, int64_t num_tokens, const int64_t *offsets,
                                      int64_t num_bags, int64_t rows, int32_t dim, int64_t first_row,
                                      int64_t padding_token, float scale, int32_t *rows_out, void *values,
                                      int32_t values_dtype, int64_t values_stride, int64_t *count, void *workspace,
                                      size_t workspace_bytes, void *stream) {
    int32_t none = 0;  // stands for the list where there are no ids: never written
    const GradCall c{Tokens{tokens, num_tokens, first_row, rows, index_type}, padding_token, offsets, num_bags, dim, scale,
                     grad_out, grad_out_dtype, grad_out_stride, values, values_dtype, values_stride, 0,
                     num_tokens > 0 ? rows_out : &none, count};
    int32_t rc = check_gradient(c);
    if (rc) return rc;
    if ((rc = check_matrix("values", values, values_dtype, values_stride, dim, dim, num_tokens))) return rc;
    if (num_tokens > 0 && !rows_out) return fail(RECMG_E_INVALID, "rows_out is NULL");
    if (reinterpret_cast<uintptr_t>(rows_out) % 4) return fail(RECMG_E_INVALID, "rows_out is not aligned to 4 bytes");
    if (!count || reinterpret_cast<uintptr_t>(count) % 8)
        return fail(RECMG_E_INVALID, "count is NULL or not aligned to 8 bytes");
    return run_gradient(c, workspace, workspace_bytes, stream);
}

}  // extern "C"
