// The products of bfloat16 operands.

#include "../../include/tt_emb.h"

#include "tt_product_kernels.h"

TT_PRODUCTS(, tt::bf16_t)
