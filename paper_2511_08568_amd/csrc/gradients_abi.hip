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
    if (l.count < 0 || l.count > kMostTensors) return fail(RECMG_E_INVALID, "num_tensors out of [0, 2^16]");
    if (l.count == 0) return RECMG_OK;
    if (!l.grads || !l.numels || !l.dtypes) return fail(RECMG_E_INVALID, "a per-tensor array is NULL");
    if (l.live_rows && !l.row_lengths) return fail(RECMG_E_INVALID, "live_rows without row_lengths");
    for (int32_t k = 0; k < l.count; ++k) {
        if (l.numels[k] < 0 || l.numels[k] > kMostElements) return fail(RECMG_E_INVALID, "numel out of [0, 2^37]");
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

// Elements per chunk of all launches of a call.
int32_t chunk_of(const Lists &l) {
    int64_t total = 0;
    for (int32_t k = 0; k < l.count; ++k) total += l.numels[k];
    int32_t chunk = kGradChunk;
    while (chunk > kLeastChunk && total / chunk < kFewChunks) chunk /= 2;
    return chunk;
}

// The next launch's tensors, from list entry *at on; false if there are none left.
bool next_launch(const Lists &l, int32_t chunk, int32_t *at, GradTensors *t) {
    t->count = t->live = t->first[0] = 0;
    t->chunk = chunk;
    t->in_place = 1;
    for (; *at < l.count && t->count < kGradTensors; ++*at) {
        const int32_t k = *at, q = t->count;
        if (l.numels[k] == 0) continue;
        if (l.live_rows && l.live_rows[k]) {
            if (t->live == kGradLive) break;
            t->live_rows[t->live] = l.live_rows[k];
            t->live_len[t->live] = l.row_lengths[k];
            t->live_of[t->live++] = (uint8_t)q;
        }
        const int64_t chunks = (l.numels[k] + chunk - 1) / chunk;
        t->src[q] = l.grads[k];
        t->dst[q] = l.outs ? l.outs[k] : nullptr;
        t->in_place &= t->src[q] == t->dst[q];
        t->tail[q] = (uint16_t)((l.numels[k] - 1) % chunk);
        t->types[q] = (uint8_t)(l.dtypes[k] + 4 * (l.outs ? l.out_dtypes[k] : 0));
        t->first[q + 1] = t->first[q] + (int32_t)chunks;
        ++t->count;
    }
    return t->count > 0;
}

int64_t most_launches(int32_t tensors) { return tensors / kGradTensors + tensors / kGradLive + 1; }

// Partial sums of all launches; returns how many.
int64_t run_sums(const Lists &l, int32_t chunk, GradTensors *t, double *partial, Launches &run) {
    int64_t launches = 0, sums = 0;
    for (int32_t at = 0; next_launch(l, chunk, &at, t);) ++launches;
    const int most = launches <= kNormLaunches ? kNormBlocks : kNormBlocksMany;
    for (int32_t at = 0; next_launch(l, chunk, &at, t);) sums += launch_norm_sums(*t, partial + sums, most, run);
    return sums;
}

int32_t check_norm(const float *norm) {
    if (!norm || reinterpret_cast<uintptr_t>(norm) % 4) return fail(RECMG_E_INVALID, "norm is NULL or not aligned to 4 bytes");
    return RECMG_OK;
}

int32_t check_limit(float max_norm, float eps) {
    if (!(max_norm >= 0.f)) return fail(RECMG_E_INVALID, "max_norm is negative or not a number");
    if (!(eps > 0.f) || eps > 1e30f) return fail(RECMG_E_INVALID, "eps out of (0, 1e30]");
    return RECMG_OK;
}

int32_t check_workspace(int32_t tensors, const void *workspace, size_t bytes) {
    size_t need = 0;
    const int32_t rc = recmg_query_grad_workspace(tensors, &need);
    if (rc) return rc;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail(RECMG_E_INVALID, "workspace is NULL or not aligned to 256 bytes");
    if (bytes < need) return fail(RECMG_E_NOMEM, "workspace smaller than recmg_query_grad_workspace says");
    return RECMG_OK;
}

}  // namespace

extern "C" {

int32_t recmg_query_grad_workspace(int32_t num_tensors, size_t *bytes) {
    if (!bytes) return fail(RECMG_E_INVALID, "bytes is NULL");
    if (num_tensors < 0 || num_tensors > kMostTensors) return fail(RECMG_E_INVALID, "num_tensors out of [0, 2^16]");
    const int64_t few = most_launches(num_tensors) < kNormLaunches ? most_launches(num_tensors) : kNormLaunches;
    const int64_t many = most_launches(num_tensors) * kNormBlocksMany;
    *bytes = (size_t)(few * kNormBlocks > many ? few * kNormBlocks : many) * sizeof(double);
    return RECMG_OK;
}

int32_t recmg_grad_norm(int32_t num_tensors, const void *const *grads, const int64_t *numels, const int32_t *dtypes,
                        const int64_t *const *live_rows, const int32_t *row_lengths, float *norm, void *workspace,
                        size_t workspace_bytes, void *stream) {
    const Lists l{num_tensors, grads, nullptr, numels, dtypes, nullptr, live_rows, row_lengths};
    int32_t rc = check_lists(l);
    if (rc || (rc = check_norm(norm)) || (rc = check_workspace(num_tensors, workspace, workspace_bytes))) return rc;
    Launches run{static_cast<hipStream_t>(stream)};
    double *partial = static_cast<double *>(workspace);
    GradTensors t;
    launch_norm_end(partial, run_sums(l, chunk_of(l), &t, partial, run), norm, run);
    return run.status();
}

int32_t recmg_grad_clip(int32_t num_tensors, const void *const *grads, void *const *outs, const int64_t *numels,
                        const int32_t *dtypes, const int32_t *out_dtypes, const int64_t *const *live_rows,
                        const int32_t *row_lengths, const float *norm, float max_norm, float eps, void *stream) {
    if (num_tensors > 0 && (!outs || !out_dtypes)) return fail(RECMG_E_INVALID, "a per-tensor array is NULL");
    const Lists l{num_tensors, grads, outs, numels, dtypes, out_dtypes, live_rows, row_lengths};
    int32_t rc = check_lists(l);
    if (rc || (rc = check_norm(norm)) || (rc = check_limit(max_norm, eps))) return rc;
    Launches run{static_cast<hipStream_t>(stream)};
    GradTensors t;
    const int32_t chunk = chunk_of(l);
    for (int32_t at = 0; next_launch(l, chunk, &at, &t);) launch_clip(t, nullptr, 0, const_cast<float *>(norm), max_norm, eps, run);
    return run.status();
}

int32_t recmg_grad_norm_clip(int32_t num_tensors, const void *const *grads, void *const *outs, const int64_t *numels,
                             const int32_t *dtypes, const int32_t *out_dtypes, const int64_t *const *live_rows,
                             const int32_t *row_lengths, float *norm, float max_norm, float eps, void *workspace,
                             size_t workspace_bytes, void *stream) {
    if (num_tensors > 0 && (!outs || !out_dtypes)) return fail(RECMG_E_INVALID, "a per-tensor array is NULL");
    const Lists l{num_tensors, grads, outs, numels, dtypes, out_dtypes, live_rows, row_lengths};
    int32_t rc = check_lists(l);
    if (rc || (rc = check_norm(norm)) || (rc = check_limit(max_norm, eps)) ||
        (rc = check_workspace(num_tensors, workspace, workspace_bytes)))
        return rc;
    Launches run{static_cast<hipStream_t>(stream)};
    double *partial = static_cast<double *>(workspace);
    GradTensors t;
    const int32_t chunk = chunk_of(l);
    const int64_t sums = run_sums(l, chunk, &t, partial, run);
    int32_t at = 0;
    const bool some = next_launch(l, chunk, &at, &t);
    // few chunks, all in one launch: the clipping kernel adds the partial sums up, one launch less
    if (some && at == l.count && t.first[t.count] <= kFusedChunks) {
        launch_clip(t, partial, sums, norm, max_norm, eps, run);
    } else {
        launch_norm_end(partial, sums, norm, run);
        for (at = 0; next_launch(l, chunk, &at, &t);) launch_clip(t, partial, 0, norm, max_norm, eps, run);
    }
    return run.status();
}

}  // extern "C"
