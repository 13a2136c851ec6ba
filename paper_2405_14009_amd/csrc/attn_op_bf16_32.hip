// Attention operator, bf16, kernels of 32 columns.
#include "attn_op_kernels.h"

hipError_t attn_op_fwd_bf16_32(const AttnOpArgs& a, hipStream_t st) { return attn_op_fwd_launch<TileB16<32>>(a, st); }
hipError_t attn_op_bwd_bf16_32(const AttnOpArgs& a, hipStream_t st) { return attn_op_bwd_launch<TileB16<32>>(a, st); }
