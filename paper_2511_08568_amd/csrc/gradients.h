// Host-side launchers of the gradient-norm and clipping kernels (gradnorm.hip);
// their C entries are in gradients_abi.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/recmg.h"

namespace recmg {

// Elements of a tensor that one block takes at a time.
constexpr int64_t kGradChunk = 16384;
// Tensors of one launch: their descriptors travel in its arguments (4 KB at most), so a
// call copies nothing to the device and may be captured into a graph.
constexpr int kGradTensors = 90;
// Blocks of one launch of the norm: a partial sum each.
constexpr int kNormBlocks = 2048;

struct GradTensors {
    const void *src[kGradTensors];
    void *dst[kGradTensors];            // clipping only
    const int64_t *live[kGradTensors];  // device count of the leading rows that hold values, or NULL: all do
    int64_t numel[kGradTensors];
    int64_t chunks;                     // of all tensors of the launch
    int32_t row_len[kGradTensors];
    int32_t first[kGradTensors];        // chunks before each tensor
    uint8_t types[kGradTensors];        // dtype of src + 4 * dtype of dst
    int32_t count;
};
static_assert(sizeof(GradTensors) <= 4096 - 64, "descriptors of one launch fit into its arguments");

// partial: the launch's kNormBlocks sums; returns how many it writes
int launch_norm_sums(const GradTensors &t, double *partial, hipStream_t s);
// the norm from the sums of all launches, kNormBlocks apart
void launch_norm_end(const double *partial, int64_t sums, float *norm, hipStream_t s);
void launch_clip(const GradTensors &t, const float *norm, float max_norm, float eps, hipStream_t s);

}  // namespace recmg
