// Low-rank adapters beside a product: what grouped.hip (its entry point) and adapters.hip (its kernels) share.
//
// Every row's inner sums, inner[m][r] = scale[g] * sum_k x[m,k] a[g,r,k], come first.  Then there are two ways:
//   fused   the product's tiles take the adapters' part into their sums (grp_adapt in grouped.h)
//   beside  the product goes to the workspace in fp32, and a last pass adds each row's part to it, column by column: where there are few rows, whose tiles
//           would wait for the loads of one adapter after another (32 rows, each with an adapter of its own, 4096 x 4096, rank 16: 53 us fused, 17 beside)
#pragma once

#include "grouped.h"

namespace alt {

struct AdapterParams {
    const char *x, *w, *a, *b;
    const int32_t *adapter;
    const float *scale, *bias;
    char *inner;
    float *base;                           // beside: the product, M x N, base_slices of them to be added
    char *y;
    int64_t ldx, ldw, ldy;                 // bytes between rows
    int32_t rows, cols, K, rank, adapters, places, relu, out_bf16;
    // what follows from these (adapters_plan)
    bool beside, few;                      // few: the product in one launch with the inner sums, beside
    int32_t inner_bytes;                   // of a row (fused: of one of its parts)
    int32_t slices, base_slices;           // beside: parts of the reductions, each with sums of its own
    int32_t slots, tiles, col_tiles;       // workgroups for a tile's adapters; tiles of rows; tiles of the rank
    int32_t few_cols;                      // column tiles of 16 to a workgroup of the product
};

void adapters_plan(int dtype, const GroupedParams &product, AdapterParams &p);
size_t adapters_inner_bytes(int dtype, const AdapterParams &p);

hipError_t adapters_down(int dtype, const AdapterParams &p, hipStream_t st);
hipError_t adapters_few(int dtype, const AdapterParams &p, hipStream_t st);
hipError_t adapters_up(int dtype, const AdapterParams &p, hipStream_t st);

}  // namespace alt
