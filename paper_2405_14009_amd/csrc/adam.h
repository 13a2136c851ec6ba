// AdamW of one element and the accesses of its streams, shared by the stage's
// step over its flat buffers and the step over many tensors.
#pragma once

#include "common.h"

namespace {

// The update lr m_hat / (sqrt(v_hat) + eps) from the new moments.  Hardware
// square root and reciprocal (1 ulp each; the update is 1e-4 of a weight, so
// their error stays far below fp32 resolution of the weight).  The rollback
// recomputes it with this same function from the same moments, so it
// subtracts exactly what the step added.
__device__ __forceinline__ float adam_update(float m, float v, float eps, float step_size,
                                             float inv_sqrt_bc2) {
  return step_size * m * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v) * inv_sqrt_bc2 + eps);
}

__device__ __forceinline__ float adam_one(float p, float g, float& m, float& v, bool decay,
                                          float lr, float b1, float b2, float eps, float wd,
                                          float step_size, float inv_sqrt_bc2, float gs) {
  g *= gs;
  m = b1 * m + (1.f - b1) * g;
  v = b2 * v + (1.f - b2) * g * g;
  if (decay) p *= (1.f - lr * wd);
  return p - adam_update(m, v, eps, step_size, inv_sqrt_bc2);
}

// The fp32 streams are read and written once per step: non-temporal accesses
// keep them from displacing cached data (-1.6 % AdamW time).
typedef float vf4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float4 ld_nt(const float4* q) {
  const vf4 t = __builtin_nontemporal_load((const vf4*)q);
  return make_float4(t.x, t.y, t.z, t.w);
}
__device__ __forceinline__ void st_nt(float4* q, float4 v) {
  const vf4 t = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(t, (vf4*)q);
}

// bf16 working copy of 4 consecutive weights: one 8-byte store.
__device__ __forceinline__ void store_bf16x4(bf16* o, float4 w) {
  const bf16 t[4] = {(bf16)w.x, (bf16)w.y, (bf16)w.z, (bf16)w.w};
  *(uint2*)o = *(const uint2*)t;
}

}  // namespace
