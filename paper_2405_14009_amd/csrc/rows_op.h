// Operators over the rows of a matrix: dropout with bias and residual, layer
// norm of such a sum, and their column sums (argument blocks and launchers).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

// A [rows, cols] matrix: columns contiguous, rows `stride` elements apart.
struct RowsView {
  void* data;
  long stride;
};

// The mask of a call: element (row, column) is kept when its 16-bit number is at
// least `threshold`, and then multiplied by `scale`.
struct DropArgs {
  int on;                 // 0: no dropout
  uint32_t threshold;     // 0 .. 65536
  float scale;            // 65536 / (65536 - threshold), 0 where nothing is kept
  uint64_t seed, offset;
  const uint64_t* step;   // device, added to offset; may be null
};

struct DropoutArgs {
  long rows;
  int cols;
  DropArgs drop;
  RowsView x, y, more;    // more: residual (added) or derivative (a factor); null data: none
  int more_factor;
  const void* bias;       // [cols], added before the mask
  int bias_f32;
  float* sums;            // [cols]: column sums of y (before rounding), or null
  int accumulate;
  float* work;
};

constexpr int NORM_MAX_COLS = 16384;

struct NormArgs {
  long rows;
  int cols;
  float eps;
  DropArgs drop;
  int params_f32;         // bias, weight and shift: fp32, else bf16
  const void *bias, *weight, *shift;  // each may be null
  RowsView x, residual, total, y;     // forward (residual, total: null data where there is none)
  float* stats;           // [2][rows]: mean, 1 / deviation; null: not stored
  RowsView dy, dtotal_in, dtotal, dx; // backward; outputs may be null, dtotal_in too
  float *dweight, *dshift, *dbias;    // fp32 [cols], each may be null
  int accumulate;
  float* work;
};

// How a matrix is shared out: lanes a row (0: whole waves), groups a lane, waves a
// row, rows side by side, workgroups.
struct NormPlan {
  int lpr, cpl, waves, slots, threads;
  long groups;
};

// Bytes of work memory for the column sums of a call.
size_t dropout_work_bytes(long rows, int cols);
size_t norm_work_bytes(long rows, int cols);
hipError_t dropout_rows(const DropoutArgs& a, int elt, hipStream_t s);
hipError_t norm_forward(const NormArgs& a, int elt, hipStream_t s);
hipError_t norm_backward(const NormArgs& a, int elt, hipStream_t s);

// out_j[c] (+)= sum over r < n of part[(r * vectors + j) * stride + c], in a fixed
// order; stride a multiple of 8.  A null out is left out.
constexpr int ROWS_MAX_VECTORS = 3;
hipError_t rows_finish(const float* part, int n, int vectors, int stride, int cols, float* const* outs, int accumulate,
                       hipStream_t s);
inline int rows_pad(int cols) { return (cols + 7) & ~7; }
