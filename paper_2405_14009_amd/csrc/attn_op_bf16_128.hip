// Attention operator, bf16, kernels of 128 columns.
#include "attn_op_kernels.h"

ATTN_OP_DEFINE(bf16_128, TileB16<128>)
