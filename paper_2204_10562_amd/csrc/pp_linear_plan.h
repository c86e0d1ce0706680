// How the products of pp_linear.hip are divided into tiles and pieces of the sum (host code, free of HIP).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "pp_layer.h"

// How a launch divides its results: ti x to tiles by `splits` pieces of the sum.  Pieces beyond one
// leave floats in `partial` [splits][outer][inner padded to 8], which k_join adds in their order.
struct pr_plan {
    long long inner, outer;
    int steps;   // of the whole sum
    int per;     // of a piece
    int splits;
    int by_piece;  // see pr_tile
    unsigned ni, no;  // tiles
    float *partial;
    long long partial_ld;
};

// bf16 planes that a gradient of this type becomes (pp_linear.hip)
static inline int planes_of(int type) { return type == PP_TYPE_BF16 ? 1 : type == PP_TYPE_F16 ? 2 : 3; }

// A tile shape: results; microseconds of a step where a compute unit has one workgroup of it and where
// it has as many as fit; how many fit; microseconds of a workgroup's start and end.  Measured: one step of
// the sum is 128 values forward and 64 in the backward products.  The estimates below choose what is within
// 9 % of the best of all shapes and numbers of pieces on 31 sizes from 16 to 32771 rows, within 4 % on 22.
// The flat shapes are for few rows: 50 rows, 4096 -> 4096 forward 12.8 us (14.1 in tiles of 128 x 128, 25.5 of
// 256 x 256, each with its best number of pieces); the large ones for many: dx of 4000 rows, 500 -> 4000 33 us (36
// in 128 x 128); for those between see the kernels.
struct pr_shape {
    int ti, to, fit;
    float alone, full, once;
};
static const pr_shape FORWARD[] = {{256, 256, 1, 1.0f, 1.0f, 12.0f}, {128, 128, 2, 0.32f, 0.62f, 6.0f}, {256, 32, 2, 0.36f, 0.5f, 5.0f}};
static const pr_shape INPUT[] = {{256, 256, 1, 1.5f, 1.7f, 12.0f}, {128, 128, 2, 0.68f, 1.14f, 7.0f}, {256, 32, 2, 0.78f, 1.1f, 5.0f}, {256, 128, 1, 0.82f, 0.9f, 8.0f}};
static const pr_shape WEIGHT[] = {{256, 256, 1, 1.5f, 1.8f, 20.0f}, {128, 128, 2, 1.0f, 1.22f, 8.0f}};
#define PR_CUS 256

// Bytes in the workspace of the partial sums, and behind them of the columns' sums of every tile of a row of tiles.
static inline size_t pr_up256(size_t x) { return (x + 255) & ~(size_t)255; }
static inline size_t partial_bytes(int pieces, long long inner, long long outer) {
    return pieces > 1 ? pr_up256((size_t)pieces * outer * ((inner + 7) & ~7ll) * 4) : 0;
}
static inline size_t sums_bytes(int pieces, long long ni, long long outer) { return pieces > 1 ? pr_up256((size_t)pieces * ni * outer * 4) : 0; }

// The shape and the number of pieces with the least estimated time: rounds of workgroups over the chip, and
// for more than one piece the pass that adds them (a launch, and each partial sum written and read).
// bi, bo: bytes of a step of the operands to an inner and an outer index.  room: bytes for the partial sums (sums: and
// the columns').  What the best number of pieces needs is not less for fewer rows (dx of 1300 rows, 16384 -> 4096, takes
// four pieces, 85 MB; of 2048 one), so a workspace sized for more rows may not hold it: then of those that fit.
#define PR_ANY_ROOM (~(size_t)0)
static inline pr_plan plan(const pr_shape *shapes, int n, long long inner, long long outer, long long steps, int bi, int bo, bool sums, size_t room,
                           int *shape) {
    pr_plan best = {};
    float least = 0;
    *shape = 0;
    for (int k = 0; k < n; ++k) {
        const pr_shape &s = shapes[k];
        const long long tiles = ((inner + s.ti - 1) / s.ti) * ((outer + s.to - 1) / s.to);
        for (int pieces = 1; pieces <= 32 && pieces <= steps; ++pieces) {
            const long long per = (steps + pieces - 1) / pieces, work = tiles * pieces;
            if (pieces > 1 && ((steps + per - 1) / per != pieces || tiles > PR_CUS * s.fit)) continue;
            if (partial_bytes(pieces, inner, outer) + (sums ? sums_bytes(pieces, (inner + s.ti - 1) / s.ti, outer) : 0) > room) break;
            const long long rounds = work / (PR_CUS * s.fit), rest = work - rounds * PR_CUS * s.fit;
            float t = (float)rounds * ((float)per * s.full + s.once);
            if (rest) t += (float)per * (rest > PR_CUS ? s.full : s.alone) + s.once;
            if (pieces > 1) t += 4.0f + (float)pieces * (0.25f + (float)(inner * outer) * 8.0f / 1.0e7f);
            if (!best.splits || t < least) {
                least = t;
                *shape = k;
                best.steps = (int)steps;
                best.per = (int)per;
                best.splits = pieces;
            }
        }
    }
    const pr_shape &s = shapes[*shape];
    // A die whose run is of one piece's tiles reads only that piece's part of the operands.  Where these are larger
    // than a few L2s (4 MiB each) that is worth it: dw of 32771 rows, 520 -> 1000 (87 MB), 69 us for 76, 8192 rows
    // (21 MB) 30 for 31; of less, reads are better spread: 2048 rows, 1024 -> 1024 (6 MB), 21.4 us for 23.7.
    best.by_piece = steps * (inner * bi + outer * bo) >= (1 << 24);
    best.inner = inner;
    best.outer = outer;
    best.ni = (unsigned)((inner + s.ti - 1) / s.ti);
    best.no = (unsigned)((outer + s.to - 1) / s.to);
    best.partial_ld = (inner + 7) & ~7ll;
    return best;
}

static inline pr_plan plan_forward(int64_t rows, int64_t n_in, int64_t n_out, size_t room, int *shape) {
    return plan(FORWARD, 3, n_out, rows, (n_in + 127) / 128, 68, 68, false, room, shape);
}
static inline pr_plan plan_input(int type, int64_t rows, int64_t n_in, int64_t n_out, size_t room, int *shape) {
    return plan(INPUT, 4, n_in, rows, planes_of(type) * ((n_out + 63) / 64), 34, 128, false, room, shape);
}
static inline pr_plan plan_weight(int type, int64_t rows, int64_t n_in, int64_t n_out, size_t room, int *shape) {
    return plan(WEIGHT, 2, n_in, n_out, planes_of(type) * (rows ? (rows + 63) / 64 : 1), 66, 128, true, room, shape);
}
