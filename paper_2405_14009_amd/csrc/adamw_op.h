// AdamW over many tensors: launcher and limits.  See adamw_op.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "recycle_stage.h"

constexpr int ADAMW_BLOCK = 128;  // elements that share a power of two (8-bit moments)

struct AdamwHyper {
  double beta1, beta2, grad_scale;  // the 32-bit arguments, widened
  float lr, weight_decay, eps;
  float step_size, inv_sqrt_bc2;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

hipError_t adamw_tensors(const rc_adamw_tensor* t, int n, int bits, const AdamwHyper& h, hipStream_t s);
