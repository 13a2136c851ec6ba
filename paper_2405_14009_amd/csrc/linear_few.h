// Products of few tokens that matrix tiles would mostly pad.
#pragma once

#include <hip/hip_runtime.h>

#include "rows_op.h"

// Most tokens that the kernel takes, by the bytes of an element: where it and the
// tile kernels meet (4096 x 4096, fp32: 16 tokens 15 and 44 us, bf16: 8 tokens 15
// and 17 us, 16 tokens 18.7 and 17.4 us).
constexpr int few_tokens_most(int elt) { return elt == 2 ? 8 : 32; }

// Rows of the gradient that a workgroup takes, and the most of them: a grid's second
// dimension holds 2^16 - 1.
constexpr int FEW_ROWS = 32, FEW_MOST_ROWS = FEW_ROWS * 0xffff;

// out [m, n] (+)= left^T right over the rows ("tokens") of both
// operands; sums, where given, (+)= the column sums of right (sums_right) or left.
// m and n multiples of 8, all rows 16-byte aligned; m at most FEW_MOST_ROWS.
struct FewTokens {
  int tokens, m, n;
  RowsView left, right;
  float *out, *sums;
  int sums_right, accumulate;
};
hipError_t few_tokens(const FewTokens& a, int elt, hipStream_t s);
