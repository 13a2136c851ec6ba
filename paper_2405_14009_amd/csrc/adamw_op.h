// AdamW over many tensors: launcher and limits.  See adamw_op.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "recycle_stage.h"

constexpr int ADAMW_BLOCK = 128;  // elements that share a power of two (8-bit moments)
// A launch holds fewer than 2^32 threads: workgroups of 256, each of at least 1024 elements.
constexpr long ADAMW_MAX_GROUPS = (1L << 24) - 1;
constexpr int64_t ADAMW_MAX_COUNT = ADAMW_MAX_GROUPS * 1024;

struct AdamwHyper {
  double beta1, beta2, grad_scale;  // the 32-bit arguments, widened
  float lr, weight_decay, eps;
  float step_size, inv_sqrt_bc2;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

AdamwHyper adamw_hyper(const rc_adam_config& a, int64_t step, float grad_scale);

hipError_t adamw_tensors(const rc_adamw_tensor* t, int n, int bits, const AdamwHyper& h, hipStream_t s);

// With 8-bit moments, read where the tensors say and written `to` bytes behind
// that (all four arrays).  undo: the parameters before that step instead, from
// the moments that it read and its gradient; no moment is written.
hipError_t adamw_banks(const rc_adamw_tensor* t, int n, const AdamwHyper& h, long to, bool undo, hipStream_t s);

hipError_t adamw_read(const rc_adamw_tensor* t, int n, int bits, float* const* m, float* const* v, hipStream_t s);

// Values of a code in a block of the given scale byte, on the host.
float adamw_decode_m(int code, int scale);
float adamw_decode_v(int code, int scale);
