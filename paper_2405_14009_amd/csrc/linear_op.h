// The linear operator's products: launches of the matrix-core kernels over the
// caller's tensors.
#pragma once

#include <hip/hip_runtime.h>

#include "rows_op.h"

struct LinearArgs {
  int elt;            // bytes an element: 2 (bf16) or 4 (fp32)
  long rows;
  int in, out;
  int by_out;         // weights [out, in] (else [in, out])
  int act;            // Act
  RowsView x, w, residual, y, slope, dy, before, dx;  // null data where there is none
  const void* bias;
  int bias_f32;
  float *dw, *dbias;  // [in, out] or [out, in]; null dbias: not formed
  int accumulate;
  void* work;
};

// Bytes of work memory: of the forward pass, the input's gradient, the weight's.
size_t linear_forward_work(const LinearArgs& a);
size_t linear_input_work(const LinearArgs& a);
size_t linear_weight_work(const LinearArgs& a);
hipError_t linear_forward(const LinearArgs& a, hipStream_t s);
hipError_t linear_backward_input(const LinearArgs& a, hipStream_t s);
hipError_t linear_backward_weight(const LinearArgs& a, hipStream_t s);
