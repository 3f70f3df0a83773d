// Layer norm and the residual step (oc_ln_*, oc_drop_ln_*): what their kernels take.
#pragma once

#include "rows.h"

namespace oc {

struct Norm {
  const void *x, *res;  // res: the residual step's, or NULL
  void *h, *y;          // h: the residual step's
  const float *gamma, *beta;
  float *mean, *invstd;
  int64_t rows;
  int c;
  bool bf16;
  float eps;
  Drop drop;
};

struct NormBwd {
  const void *x, *res, *dy, *dh;  // h = res + dropout(x) is formed again
  void *dx, *dres;  // dx: behind the dropout; dres: in front of it (a plain norm's dx)
  const float *gamma, *mean, *invstd;
  float* delta;  // [rows], times invstd, for the column sums of rows too long for registers
  int64_t rows;
  int c;
  bool bf16;
  Drop drop;
};

// Sums over rows: at most this many are added in fp32, the rest in double.
constexpr int64_t MOST_ADDED = 64;

// Rows that fit a workgroup's registers (norm_rows.hip).
constexpr int32_t NORM_ROWS_MOST = 16384;
void norm_rows_fwd(const Norm& a, hipStream_t s);
// part: [norm_rows_blocks()][2][c] sums of the workgroups' rows, or NULL.
int64_t norm_rows_blocks(int64_t rows, int32_t c);
void norm_rows_bwd(const NormBwd& a, float* part, hipStream_t s);

}  // namespace oc
