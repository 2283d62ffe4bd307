// C entries of the norm of many gradients and their clipping.
#include "gradients.h"
#include "status.h"
#include "values.h"

using namespace recmg;

namespace {

// What both entries take of the tensors; outs and out_dtypes NULL where nothing is written.
struct Lists {
    int32_t count;
    const void *const *grads;
    void *const *outs;
    const int64_t *numels;
    const int32_t *dtypes, *out_dtypes;
    const int64_t *const *live_rows;
    const int32_t *row_lengths;
};

bool bad_dtype(int32_t d) { return d != RECMG_F32 && d != RECMG_F16 && d != RECMG_BF16; }

int32_t check_lists(const Lists &l) {
    if (l.count < 0 || l.count > (1 << 20)) return fail(RECMG_E_INVALID, "num_tensors out of [0, 2^20]");
    if (l.count == 0) return RECMG_OK;
    if (!l.grads || !l.numels || !l.dtypes) return fail(RECMG_E_INVALID, "a per-tensor array is NULL");
    if (l.live_rows && !l.row_lengths) return fail(RECMG_E_INVALID, "live_rows without row_lengths");
    for (int32_t k = 0; k < l.count; ++k) {
        if (l.numels[k] < 0 || l.numels[k] > (int64_t(1) << 40)) return fail(RECMG_E_INVALID, "numel out of [0, 2^40]");
        if (bad_dtype(l.dtypes[k])) return fail(RECMG_E_INVALID, "bad dtype");
        if (l.numels[k] == 0) continue;
        if (!l.grads[k]) return fail(RECMG_E_INVALID, "a gradient is NULL");
        if (reinterpret_cast<uintptr_t>(l.grads[k]) % elem_size(l.dtypes[k]))
            return fail(RECMG_E_INVALID, "a gradient is not aligned to its elements");
        if (l.live_rows && l.live_rows[k]) {
            if (l.row_lengths[k] < 1) return fail(RECMG_E_INVALID, "row_lengths entry below 1");
            if (reinterpret_cast<uintptr_t>(l.live_rows[k]) % 8)
                return fail(RECMG_E_INVALID, "a live_rows count is not aligned to 8 bytes");
        }
        if (l.outs) {
            const int32_t od = l.out_dtypes[k];
            if (bad_dtype(od)) return fail(RECMG_E_INVALID, "bad out dtype");
            if (!l.outs[k]) return fail(RECMG_E_INVALID, "an output is NULL");
            if (reinterpret_cast<uintptr_t>(l.outs[k]) % elem_size(od))
                return fail(RECMG_E_INVALID, "an output is not aligned to its elements");
            if (l.outs[k] == l.grads[k] && od != l.dtypes[k])
                return fail(RECMG_E_INVALID, "an output in place of its gradient must have its dtype");
        }
    }
    return RECMG_OK;
}

// The next launch's tensors, from list entry *at on; false if there are none left.
bool next_launch(const Lists &l, int32_t *at, GradTensors *t) {
    t->count = 0;
    t->chunks = 0;
    for (; *at < l.count && t->count < kGradTensors; ++*at) {
        const int32_t k = *at;
        if (l.numels[k] == 0) continue;
        const int64_t chunks = (l.numels[k] + kGradChunk - 1) / kGradChunk;
        if (t->count > 0 && t->chunks + chunks >= (int64_t(1) << 31)) break;  // at most 2^26 of one tensor
        const int32_t q = t->count++;
        t->src[q] = l.grads[k];
        t->dst[q] = l.outs ? l.outs[k] : nullptr;
        t->live[q] = l.live_rows ? l.live_rows[k] : nullptr;
        t->numel[q] = l.numels[k];
        t->row_len[q] = t->live[q] ? l.row_lengths[k] : 1;
        t->first[q] = (int32_t)t->chunks;
        t->types[q] = (uint8_t)(l.dtypes[k] + 4 * (l.outs ? l.out_dtypes[k] : 0));
        t->chunks += chunks;
    }
    return t->count > 0;
}

}  // namespace

extern "C" {

int32_t recmg_query_grad_workspace(int32_t num_tensors, size_t *bytes) {
    if (!bytes) return fail(RECMG_E_INVALID, "bytes is NULL");
    if (num_tensors < 0 || num_tensors > (1 << 20)) return fail(RECMG_E_INVALID, "num_tensors out of [0, 2^20]");
    // launches: full ones, and one more wherever one ends early for its number of chunks
    const int64_t launches = (num_tensors + kGradTensors - 1) / kGradTensors + num_tensors / 31 + 1;
    *bytes = (size_t)launches * kNormBlocks * sizeof(double);
    return RECMG_OK;
}

int32_t recmg_grad_norm(int32_t num_tensors, const void *const *grads, const int64_t *numels, const int32_t *dtypes,
                        const int64_t *const *live_rows, const int32_t *row_lengths, float *norm, void *workspace,
                        size_t workspace_bytes, void *stream) {
    const Lists l{num_tensors, grads, nullptr, numels, dtypes, nullptr, live_rows, row_lengths};
    int32_t rc = check_lists(l);
    if (rc) return rc;
    if (!norm || reinterpret_cast<uintptr_t>(norm) % 4) return fail(RECMG_E_INVALID, "norm is NULL or not aligned to 4 bytes");
    size_t need = 0;
    if ((rc = recmg_query_grad_workspace(num_tensors, &need))) return rc;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail(RECMG_E_INVALID, "workspace is NULL or not aligned to 256 bytes");
    if (workspace_bytes < need) return fail(RECMG_E_NOMEM, "workspace smaller than recmg_query_grad_workspace says");
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *partial = static_cast<double *>(workspace);
    GradTensors t;
    int64_t sums = 0;
    for (int32_t at = 0; next_launch(l, &at, &t);) sums += launch_norm_sums(t, partial + sums, s);
    launch_norm_end(partial, sums, norm, s);
    HIP_TRY(hipGetLastError());
    return RECMG_OK;
}

int32_t recmg_grad_clip(int32_t num_tensors, const void *const *grads, void *const *outs, const int64_t *numels,
                        const int32_t *dtypes, const int32_t *out_dtypes, const int64_t *const *live_rows,
                        const int32_t *row_lengths, const float *norm, float max_norm, float eps, void *stream) {
    if (num_tensors > 0 && (!outs || !out_dtypes)) return fail(RECMG_E_INVALID, "a per-tensor array is NULL");
    const Lists l{num_tensors, grads, outs, numels, dtypes, out_dtypes, live_rows, row_lengths};
    const int32_t rc = check_lists(l);
    if (rc) return rc;
    if (!norm || reinterpret_cast<uintptr_t>(norm) % 4) return fail(RECMG_E_INVALID, "norm is NULL or not aligned to 4 bytes");
    if (!(max_norm >= 0.f)) return fail(RECMG_E_INVALID, "max_norm is negative or not a number");
    if (!(eps > 0.f) || eps > 1e30f) return fail(RECMG_E_INVALID, "eps out of (0, 1e30]");
    hipStream_t s = static_cast<hipStream_t>(stream);
    GradTensors t;
    for (int32_t at = 0; next_launch(l, &at, &t);) launch_clip(t, norm, max_norm, eps, s);
    HIP_TRY(hipGetLastError());
    return RECMG_OK;
}

}  // extern "C"
