// Launches of the layer norm operator (kernels: norm_op_kernels.h).
#include <algorithm>

#include "common.h"
#include "rows_op.h"

hipError_t norm_fwd_bf16(const NormPlan& p, const NormArgs& a, hipStream_t s);
hipError_t norm_fwd_f32(const NormPlan& p, const NormArgs& a, hipStream_t s);
hipError_t norm_bwd_bf16(const NormPlan& p, const NormArgs& a, hipStream_t s);
hipError_t norm_bwd_f32(const NormPlan& p, const NormArgs& a, hipStream_t s);

namespace {

constexpr int CUS = 256;   // compute units that grids are sized for

// sums: the columns' sums are kept, of which each workgroup stores a row: as few
// workgroups as fill the card, with several rows side by side in each.
NormPlan plan_of(long rows, int cols, bool sums) {
  NormPlan p{};
  const int groups = (cols + 7) / 8;
  p.waves = 1;
  p.threads = 256;
  if (cols <= 1024) {
    p.lpr = cols <= 32 ? 4 : cols <= 128 ? 16 : 64;
    p.cpl = cols <= 512 ? 1 : 2;
    p.slots = 256 / p.lpr;
  } else {
    p.lpr = 0;
    p.cpl = groups <= 1024 ? 1 : 2;
    p.waves = (groups + 64 * p.cpl - 1) / (64 * p.cpl);
    p.slots = sums ? std::max(1, 16 / p.waves) : 1;
    p.threads = 64 * p.waves * p.slots;
  }
  const long sets = std::max(1L, (rows + p.slots - 1) / p.slots);
  // Threads that a compute unit's share of the grid has: four waves a SIMD with sums,
  // else seven, what the forward of bf16 rows of 1025 .. 8192 columns, in whole
  // groups, holds at a time.  The other kernels hold fewer (odd bf16 rows six, fp32 rows five or
  // four, 513 .. 1024 columns four or three and backward two, a backward pass without
  // sums four), so that a full grid of theirs walks its rows in a second, partly empty
  // round of workgroups.
  const int room = sums ? 1024 : 1792;
  // sums of few rows are one workgroup's, which stores them itself
  if (sums && sets <= 4) p.groups = 1;
  else p.groups = std::min(sets, (long)CUS * std::max(1, room / p.threads));
  return p;
}

}  // namespace

size_t norm_work_bytes(long rows, int cols) {
  const long groups = plan_of(rows, cols, true).groups;
  return groups > 1 ? sizeof(float) * (size_t)groups * ROWS_MAX_VECTORS * rows_pad(cols) : 0;
}

hipError_t norm_forward(const NormArgs& a, int elt, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const NormPlan p = plan_of(a.rows, a.cols, false);
  return elt == 2 ? norm_fwd_bf16(p, a, s) : norm_fwd_f32(p, a, s);
}

hipError_t norm_backward(const NormArgs& a, int elt, hipStream_t s) {
  const bool sums = a.dweight || a.dshift || a.dbias;
  if (a.rows == 0 && !sums) return hipSuccess;
  const NormPlan p = plan_of(a.rows, a.cols, sums);
  const hipError_t e = elt == 2 ? norm_bwd_bf16(p, a, s) : norm_bwd_f32(p, a, s);
  if (e != hipSuccess || !sums || p.groups == 1) return e;
  float* const outs[3] = {a.dweight, a.dshift, a.dbias};
  return rows_finish(a.work, (int)p.groups, 3, rows_pad(a.cols), a.cols, outs, a.accumulate, s);
}
