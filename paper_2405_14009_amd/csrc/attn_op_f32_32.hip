// Attention operator, fp32, kernels of 32 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(f32_32, TileF32<32>)
