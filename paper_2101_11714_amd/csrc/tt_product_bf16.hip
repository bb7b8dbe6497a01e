// The products of bfloat16 operands.

#include "../../include/tt_emb.h"

#include "tt_product_kernels.h"

template int tt::product_of<tt::bf16_t>(tt::Layout, int32_t, const tt::Operand &, const tt::Operand &, int64_t, int64_t, int64_t, const tt::EpilogueArgs &, void *, hipStream_t);
