// The products of 32-bit operands.

#include "../../include/tt_emb.h"

#include "tt_product_kernels.h"

TT_PRODUCTS(, float)
