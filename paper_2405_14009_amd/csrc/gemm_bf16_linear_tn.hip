// bf16 GEMMs of the linear operator with both operands m/n-contiguous: weight
// gradients of weights [out, in], which sum the columns of their left operand (dy).
#include "gemm_bf16_tile.h"

hipError_t gemm_bf16_linear_tn(const GemmParams& p, hipStream_t s) {
  if (p.epi != EPI_F32_ACC) return hipErrorInvalidValue;
  return launch_bf16<false, false, EPI_F32_ACC, true>(p, s);
}
