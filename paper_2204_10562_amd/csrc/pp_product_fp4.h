// Products of two packed matrices in blocks of 4 bits (pp_product_fp4.hip).
#pragma once
#include "pp_product.h"

struct p4_operands {
    const uint8_t *inner_codes, *inner_scales, *outer_codes, *outer_scales;
};
int p4_launch(int shape, int type, const pr_plan &p, const p4_operands &q, void *y, long long ld, const float *bias, hipStream_t st);
