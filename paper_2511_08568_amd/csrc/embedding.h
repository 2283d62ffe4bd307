// Host-side launchers of the token-embedding kernels: the lookup (lookup.hip),
// its gradient (rowgrad.hip); their C entries are in embedding_abi.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/recmg.h"
#include "status.h"

namespace recmg {

// Token ids and the part of them that a table (or its gradient) holds.
struct Tokens {
    const void *ids;
    int64_t n, first_row, rows;
    int32_t index_type;
};

void launch_lookup(const void *table, int32_t table_dtype, int64_t table_stride, const Tokens &tok, int32_t dim,
                   float scale, void *out, int32_t out_dtype, int64_t out_stride, Launches &run);

// ---- gradient: ids sorted by row, then the rows' sums ----

// Whole-table gradients of so few ids, and of so few values, are made by one kernel: its blocks compare the ids once per
// 512 columns.  One kernel against sorting and summing: 20,000 x 1,024 bf16, 1,024 ids 10.6 us, 20.7; 1,500 ids 16.6,
// 21.1; 2,048 ids 23.6, 20.9.  50,000 x 4,096, 512 ids 18.1, 20.2; 1,024 ids 40.4, 20.3.  50,000 x 256 fp32, 2,048 ids
// 12.3, 20.4, and 32.7, 20.6 where all are one row.
constexpr int kDirectIds = 2048;
constexpr int64_t kDirectFew = 512, kDirectValuesFew = 4096 * 512, kDirectValues = 3000 * 512;
// In the rows form a block of that kernel also counts the distinct rows below its own: up to so many ids, and ids squared
// times columns.  One kernel against sorting and summing: 64 ids 8.4 us, 18; 128 ids of 4,096 bf16 columns 13.4, 19.7; 256
// ids of 1,024 columns 17.6, 20; of 4,096 columns 37, 19.7.
constexpr int64_t kDirectRows = 256, kDirectRowsWork = 256 * 256 * 1024;
// Ids up to which comparisons sort them, instead of radix passes: 50,000 x 256 fp32, 8,192 ids 28 us, 45; 12,000 ids 42,
// 46, but 60, 44 where all are one row.
constexpr int kRankIds = 8 * 1024;
constexpr int kSortTile = 4096;   // ids per block of the radix sort
constexpr int kMaxDigit = 10;     // bits a pass of it goes by, at most

// How one call sorts and sums, and where its arrays lie in the workspace.
struct GradPlan {
    bool direct, ranked;
    int32_t ntiles, passes, digit;      // digit: bits per pass
    int32_t chunk;                      // sorted ids whose sums one group of lanes makes
    int64_t nchunk;
    size_t ids[2], cnt, tot, ccnt, hcnt, part, total;
};
GradPlan grad_plan(int64_t rows, int32_t dim, int64_t n, bool rows_form, bool bags);

struct GradCall {
    Tokens tok;
    int64_t padding_token;             // an id without a gradient
    const int64_t *offsets;            // bags, or NULL: one row of grad_out per id
    int64_t num_bags;
    int32_t dim;
    float scale;
    const void *grad_out;
    int32_t grad_out_dtype;
    int64_t grad_out_stride;
    void *grad;                        // rows form: the values
    int32_t grad_dtype;
    int64_t grad_stride;
    int32_t accumulate;                // the whole table's gradient only
    int32_t *rows_out;                 // rows form: distinct rows, else NULL
    int64_t *count;
};
void launch_row_gradient(const GradCall &c, const GradPlan &p, char *workspace, Launches &run);

}  // namespace recmg
