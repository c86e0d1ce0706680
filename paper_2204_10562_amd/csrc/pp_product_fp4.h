// Products of two packed matrices in blocks of 4 bits (pp_product_fp4.hip).
#pragma once
#include "pp_product.h"

struct p4_operands {
    const uint8_t *inner_codes, *inner_scales, *outer_codes, *outer_scales;
};
int p4_launch(int shape, int type, const pr_plan &p, const p4_operands &q, void *y, long long ld, const float *bias, hipStream_t st);

// Few rows, where r4_takes says so: with x packed as q's outer operand, or, where r4_fuses says so, x itself.
bool r4_takes(int64_t rows, int64_t n_in, int64_t n_out);
bool r4_fuses(int64_t rows, int64_t n_in);
int r4_launch(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *x, int64_t ld_x, uint8_t *kept_codes, uint8_t *kept_scales,
              const p4_operands &q, void *y, int64_t ld_y, const float *bias, hipStream_t st);
