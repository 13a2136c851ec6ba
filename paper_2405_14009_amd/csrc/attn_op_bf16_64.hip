// Attention operator, bf16, kernels of 64 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(bf16_64, TileB16<64>)
