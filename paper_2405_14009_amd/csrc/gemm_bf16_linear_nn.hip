// bf16 GEMMs of the linear operator with A k-contiguous and B n-contiguous: its
// forward pass (weights [in, out]) and, with weights [out, in], its input gradient
// times the derivative of the activation before.
#include "gemm_bf16_tile.h"

hipError_t gemm_bf16_linear_nn(const GemmParams& p, hipStream_t s) {
  switch (p.epi) {
    case EPI_LINEAR: return launch_bf16<true, false, EPI_LINEAR>(p, s);
    case EPI_GELU_BWD: return launch_bf16<true, false, EPI_GELU_BWD>(p, s);
    default: return hipErrorInvalidValue;
  }
}
