// The products of float16 operands.

#include "../../include/tt_emb.h"

#include "tt_product_kernels.h"

TT_PRODUCTS(, tt::f16_t)
