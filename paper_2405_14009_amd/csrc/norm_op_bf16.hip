#include "norm_op_kernels.h"

hipError_t norm_fwd_bf16(const NormPlan& p, const NormArgs& a, hipStream_t s) { return norm_fwd<bf16>(p, a, s); }
hipError_t norm_bwd_bf16(const NormPlan& p, const NormArgs& a, hipStream_t s) { return norm_bwd<bf16>(p, a, s); }
