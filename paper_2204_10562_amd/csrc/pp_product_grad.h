// Products of gradients with a packed operand (pp_product_grad.hip).
#pragma once
#include "pp_product.h"

// The outer operand in bf16 as `planes` matrices that add up to it (one, or more where its type has
// more bits), `plane` values apart, each of rows x cols with rows ld values apart; every row starts
// at a multiple of 16 bytes.  What lies between a row's end and the next row is not used.  cols is a
// multiple of 8 for pg_launch_input, whose sum runs along the rows, and even for pg_launch_weight.
struct pg_outer {
    const uint8_t *p;
    long long rows, cols, ld, plane;
    int planes;
};
// The packed inner operand, whose rows the sum runs over.
struct pg_inner {
    const uint8_t *codes, *scales;
    long long rows, groups;
};
int pg_launch_input(int shape, int type, const pr_plan &p, const pg_inner &w, const pg_outer &dy, void *dx, long long ld, hipStream_t st);
int pg_launch_weight(int shape, const pr_plan &p, const pg_inner &x, const pg_outer &dy, float *dw, long long ld, const float *add, float *sums,
                     hipStream_t st);
