// Attention operator, fp32, kernels of 128 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(f32_128, TileF32<128>)
