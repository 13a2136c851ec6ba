// bf16 GEMMs of the linear operator with both operands k-contiguous: its forward
// pass with weights [out, in].
#include "gemm_bf16_tile.h"

hipError_t gemm_bf16_linear_nt(const GemmParams& p, hipStream_t s) {
  if (p.epi != EPI_LINEAR) return hipErrorInvalidValue;
  return launch_bf16<true, true, EPI_LINEAR>(p, s);
}
