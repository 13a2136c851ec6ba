#include "norm_op_kernels.h"

hipError_t norm_fwd_bf16(const NormArgs& a, hipStream_t s) { return norm_fwd<bf16>(a, s); }
hipError_t norm_bwd_bf16(const NormArgs& a, int groups, hipStream_t s) { return norm_bwd<bf16>(a, groups, s); }
