// Products of the dense gated feed-forward with few rows.  Internal to libcep.
#pragma once

#include "common.h"

namespace cep {

// Whether, and how, a forward pass of `rows` rows streams the weights in row
// blocks (dense_rows.hip) instead of running the tiled product (dense.hip).
struct RowsPlan {
  bool use;
  int splits1, splits2;  // K shares of the two products
};
RowsPlan rows_plan(int rows, int d, int I);
// Bytes of its scratch.
size_t rows_workspace(const RowsPlan &p, int rows, int d, int I);
void launch_rows_ffn(const RowsPlan &p, int rows, int d, int I, const __bf16 *x, int64_t ld_x,
                     const __bf16 *wg, const __bf16 *wu, const __bf16 *wd, __bf16 *y, int64_t ld_y,
                     float *pre, uint8_t *workspace, hipStream_t s);

}  // namespace cep
