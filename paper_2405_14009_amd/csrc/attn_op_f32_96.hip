// Attention operator, fp32, kernels of 96 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(f32_96, TileF32<96>)
