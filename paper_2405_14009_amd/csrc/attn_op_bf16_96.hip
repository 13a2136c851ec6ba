// Attention operator, bf16, kernels of 96 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(bf16_96, TileB16<96>)
