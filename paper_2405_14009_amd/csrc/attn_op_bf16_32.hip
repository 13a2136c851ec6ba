// Attention operator, bf16, kernels of 32 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(bf16_32, TileB16<32>)
