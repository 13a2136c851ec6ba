// Products of few tokens that matrix tiles would mostly pad.
#pragma once

#include <hip/hip_runtime.h>

#include "rows_op.h"

// Most tokens that the kernel takes, by the bytes of an element.  bf16: where it and
// the tile kernels meet (4096 x 4096: 8 tokens 15 and 19 us, 16 tokens 18.7 and 17.4
// to 19).  fp32: what a thread holds of them in registers (176 of 32 tokens; 4096 x
// 4096: 16 tokens 15 and 39 us, 32 tokens 22 and 39), which is short of where the two
// would meet.
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
