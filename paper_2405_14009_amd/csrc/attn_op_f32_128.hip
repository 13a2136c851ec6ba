// Attention operator, fp32, kernels of 128 columns.
#include "attn_op_kernels.h"

hipError_t attn_op_fwd_f32_128(const AttnOpArgs& a, hipStream_t st) { return attn_op_fwd_launch<TileF32<128>>(a, st); }
hipError_t attn_op_bwd_f32_128(const AttnOpArgs& a, hipStream_t st) { return attn_op_bwd_launch<TileF32<128>>(a, st); }
