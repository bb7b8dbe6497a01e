// The products of 32-bit operands.

#include "../../include/tt_emb.h"

#include "tt_product_kernels.h"

template int tt::product_of<float>(tt::Layout, int32_t, const tt::Operand &, const tt::Operand &, int64_t, int64_t, int64_t, const tt::EpilogueArgs &, void *, hipStream_t);
