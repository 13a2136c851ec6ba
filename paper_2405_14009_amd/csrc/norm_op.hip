// Launches of the layer norm operator (kernels: norm_op_kernels.h).
#include <algorithm>

#include "norm_op_kernels.h"

namespace {

int lanes_of(int cols) { return cols <= 32 ? 4 : cols <= 128 ? 16 : cols <= 1024 ? 64 : cols <= 4096 ? 256 : cols <= 8192 ? 512 : 1024; }

// Workgroups of the backward pass: two of 256 threads a compute unit where column
// sums are kept (each stores a row of them), else one a set of rows.
long groups_of(long rows, int cols, bool sums) {
  const int lanes = lanes_of(cols), per = block_of(lanes) / lanes;
  const long all = std::max(1L, (rows + per - 1) / per);
  return std::min(all, sums ? 512L * 256 / block_of(lanes) : 1L << 20);
}

}  // namespace

size_t norm_work_bytes(long rows, int cols, int) {
  return sizeof(float) * (size_t)groups_of(rows, cols, true) * ROWS_MAX_VECTORS * rows_pad(cols);
}

hipError_t norm_forward(const NormArgs& a, int elt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return elt == 2 ? norm_fwd_bf16(a, s) : norm_fwd_f32(a, s);
}

hipError_t norm_backward(const NormArgs& a, int elt, hipStream_t s) {
  const bool sums = a.dweight || a.dshift || a.dbias;
  if (a.rows == 0 && !sums) return hipSuccess;
  const int groups = (int)groups_of(a.rows, a.cols, sums);
  const hipError_t e = elt == 2 ? norm_bwd_bf16(a, groups, s) : norm_bwd_f32(a, groups, s);
  if (e != hipSuccess || !sums) return e;
  float* const outs[3] = {a.dweight, a.dshift, a.dbias};
  return rows_finish(a.work, groups, 3, rows_pad(a.cols), a.cols, outs, a.accumulate, s);
}
