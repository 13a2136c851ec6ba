// Attention operator, fp32, kernels of 64 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(f32_64, TileF32<64>)
