#include "norm_op_kernels.h"

hipError_t norm_fwd_f32(const NormPlan& p, const NormArgs& a, hipStream_t s) { return norm_fwd<float>(p, a, s); }
hipError_t norm_bwd_f32(const NormPlan& p, const NormArgs& a, hipStream_t s) { return norm_bwd<float>(p, a, s); }
