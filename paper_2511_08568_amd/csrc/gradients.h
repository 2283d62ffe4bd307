// Host-side launchers of the gradient-norm and clipping kernels (gradnorm.hip);
// their C entries are in gradients_abi.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/recmg.h"
#include "status.h"

namespace recmg {

// Elements of a tensor that one block takes at a time: fewer where there would be fewer than kFewChunks chunks, so that
// short calls use the whole chip (norm and clipping of 62 tensors of 2 million elements: 14.6 us with 16,384, 12.8 with
// 2,048).
constexpr int32_t kGradChunk = 16384, kLeastChunk = 2048;
constexpr int64_t kFewChunks = 1024;
// Tensors of one launch, and those among them with a count: their descriptors travel in its arguments (4 KB at
// most), so a call copies nothing to the device and may be captured into a graph.
constexpr int kGradTensors = 160, kGradLive = 20;
// Blocks of one launch of the norm (a partial sum each): those of calls of up to kNormLaunches launches, of more.
constexpr int kNormBlocks = 2048, kNormBlocksMany = 256, kNormLaunches = 16;
// Up to so many chunks the clipping kernel's blocks add up the partial sums themselves, each for itself.
constexpr int64_t kFusedChunks = 2048;
constexpr int64_t kMostTensors = 1 << 16, kMostElements = int64_t(1) << 37;  // of a call, of a tensor
static_assert((int64_t)kGradTensors * (kMostElements / kGradChunk) < (int64_t(1) << 31), "chunks of a launch are counted in 32 bits");

struct GradTensors {
    const void *src[kGradTensors];
    void *dst[kGradTensors];               // clipping only
    const int64_t *live_rows[kGradLive];   // device counts of the leading rows that hold values
    int32_t live_len[kGradLive];           // elements of such a row
    int32_t first[kGradTensors + 1];       // chunks before each tensor; the last: of all
    uint16_t tail[kGradTensors];           // elements of the last chunk, less one
    uint8_t types[kGradTensors];           // dtype of src + 4 * dtype of dst
    uint8_t live_of[kGradLive];            // the tensors that live_rows belong to
    int32_t count, live, chunk, in_place;  // in_place: every dst is its src
};
static_assert(sizeof(GradTensors) <= 4096 - 64, "descriptors of one launch fit into its arguments");

// partial: at least `most` sums; returns how many it writes
int launch_norm_sums(const GradTensors &t, double *partial, int most, Launches &run);
// the norm from the partial sums of all launches; in 64 bits it replaces the first of them
void launch_norm_end(double *partial, int64_t sums, float *norm, Launches &run);
// sums > 0: the norm from these partial sums, written to norm too; else it is read, from partial[0] in 64 bits, or from
// norm where partial is NULL
void launch_clip(const GradTensors &t, const double *partial, int64_t sums, float *norm, float max_norm, float eps,
                 Launches &run);

}  // namespace recmg
