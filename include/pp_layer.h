/*
 * pp_layer.h - operators of the layers that a pipeline stage runs, on one MI355X.
 *
 * Part of libpp (hand-written HIP kernels for gfx950).  The planner of pp.h takes, for every
 * layer, the times of a microbatch's forward and backward pass and the bytes that cross a cut;
 * a synchronous pipeline keeps those bytes for every microbatch until its backward pass.  The
 * operators here hold such activations in 8 bits and read them as they are in the backward
 * pass, and multiply linear layers' operands in 4 bits.
 *
 * General rules
 *   - The rules of pp.h hold: device pointers, the caller owns every buffer, no allocation, no
 *     state between calls, no synchronisation, all work on `stream`; PP_OK or a negative
 *     PP_ERR_* with nothing enqueued.  Results are the same bit for bit from call to call.
 *   - `type` is PP_TYPE_F32, _F16 or _BF16.  A matrix has rows of `cols` consecutive values,
 *     `ld` values apart (ld >= cols; ld is not read where there is one row); its base has its
 *     type's alignment.  rows >= 0 (0: nothing is enqueued but what has to be written all the
 *     same), 1 <= cols <= PP_LAYER_MAX_COLS, rows <= PP_LAYER_MAX_ROWS.
 *   - Inputs and outputs must not overlap unless said otherwise.
 *   - Sums and the functions are computed in 32 bits and rounded once, to the nearest.
 *
 * Packed matrix of R rows and C columns: G = ceil(C / 128) groups to a row.
 *   PP_PACK_INT8  codes int8  [R][G][128]
 *   PP_PACK_FP4   codes uint8 [R][G][64], two E2M1 values to a byte, the even column's low
 *   scales        uint8 [R][G][4], one per block of 32 columns
 * Codes and scales start at a multiple of 16 bytes.  What lies beyond column C has code 0, and
 * a block with no column scale 0.  For a block with a = max |v| and e = floor(log2 a), -127 for
 * smaller ones and zero:
 *   INT8  scale byte e + 127, code = 64 v / 2^e to the nearest (ties to even), at most 127 in
 *         size, value = code * 2^(byte - 133)
 *   FP4   scale byte max(e - 2 + 127, 0), code = v / 2^(byte - 127) to the nearest of 0 .5 1 1.5
 *         2 3 4 6 and their negatives (ties to the even code; 6 beyond 6; the sign of what
 *         rounds to zero is kept), value = code * 2^(byte - 127)
 * A block that holds a NaN or an infinity has scale byte 255 and codes 0: all of it reads NaN.
 */
#ifndef PP_LAYER_H
#define PP_LAYER_H

#include "pp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PP_TYPE_F32 0
#define PP_TYPE_F16 1
#define PP_TYPE_BF16 2

#define PP_PACK_INT8 0
#define PP_PACK_FP4 1

#define PP_ACT_GELU 0      /* x Phi(x)                                          */
#define PP_ACT_GELU_TANH 1 /* x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2   */
#define PP_ACT_SILU 2      /* x / (1 + exp(-x))                                 */

#define PP_LAYER_MAX_ROWS (1 << 30)
#define PP_LAYER_MAX_COLS (1 << 22)
#define PP_LAYER_MAX_LD_DW (1 << 24)

/* src [rows][cols] -> packed. */
int pp_pack(int format, int type, int64_t rows, int64_t cols, const void *src, int64_t ld_src, void *codes,
            void *scales, void *stream);

/* packed -> dst [rows][cols], rounded to `type`. */
int pp_unpack(int format, int type, int64_t rows, int64_t cols, const void *codes, const void *scales, void *dst,
              int64_t ld_dst, void *stream);

/*
 * Activation function, forward, in one pass over x (and u):
 *   y = f(x), or f(x) * u where u is given (a gated layer);
 *   x (and u) packed with PP_PACK_INT8, for pp_act_backward.
 *   x, u, y          [rows][cols], all of `type`; u NULL = not gated
 *   x_codes/x_scales, u_codes/u_scales   out, or NULL = not kept (both of a pair, or none;
 *                    u's only with u)
 */
int pp_act_forward(int kind, int type, int64_t rows, int64_t cols, const void *x, int64_t ld_x, const void *u,
                   int64_t ld_u, void *y, int64_t ld_y, void *x_codes, void *x_scales, void *u_codes, void *u_scales,
                   void *stream);

/*
 * Its backward pass from the kept values xk (and uk):
 *   dx = dy f'(xk), or dy f'(xk) uk;   du = dy f(xk)
 *   dy, dx, du       [rows][cols], all of `type`; dx may be dy (same base and ld) where du is NULL
 *   u_codes/u_scales and du  all NULL = not gated
 */
int pp_act_backward(int kind, int type, int64_t rows, int64_t cols, const void *dy, int64_t ld_dy, const void *x_codes,
                    const void *x_scales, const void *u_codes, const void *u_scales, void *dx, int64_t ld_dx, void *du,
                    int64_t ld_du, void *stream);

/*
 * The linear layer y = x W^T + b with its weight W [n_out][n_in] packed with PP_PACK_FP4.
 * pp_linear_workspace_bytes: bytes of workspace that the call of this kind needs (host function;
 * 0 if a size or the type is out of range).  What a type needs serves the types of fewer bits too, and
 * what so many rows need serves fewer.  (Fewer rows may want more bytes, for the partial sums of a sum
 * that is divided into more pieces: a call divides its sum as its workspace allows, so with less than
 * it asks for its results may be rounded otherwise, and it may take longer.  From these bytes on, more
 * change nothing.)  The workspace must be 256-byte aligned; its contents need not be kept.
 */
#define PP_LINEAR_FORWARD 0
#define PP_LINEAR_BACKWARD_INPUT 1
#define PP_LINEAR_BACKWARD_WEIGHT 2
size_t pp_linear_workspace_bytes(int call, int type, int64_t rows, int64_t n_in, int64_t n_out);

/*
 * y = q(x) W^T + b, where q(x) is x packed with PP_PACK_FP4 and read back.
 *   x [rows][n_in], y [rows][n_out] of `type`; bias float [n_out] or NULL
 *   x_codes, x_scales  out: x packed with PP_PACK_INT8 for pp_linear_backward_weight, or both NULL
 */
int pp_linear_forward(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *x, int64_t ld_x,
                      const void *w_codes, const void *w_scales, const float *bias, void *y, int64_t ld_y,
                      void *x_codes, void *x_scales, void *workspace, size_t workspace_bytes, void *stream);

/* dx = dy W: dy [rows][n_out], dx [rows][n_in] of `type`. */
int pp_linear_backward_input(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *dy, int64_t ld_dy,
                             const void *w_codes, const void *w_scales, void *dx, int64_t ld_dx, void *workspace,
                             size_t workspace_bytes, void *stream);

/*
 * dw = dw_in + dy^T xk, db = sum over the rows of dy, with xk the kept x (PP_PACK_INT8).  (The forward pass
 * multiplied x in 4 bits; xk is nearer to x than that, so dw is the gradient of x W^T, with rounding passed
 * straight through, and not the derivative of what the forward pass computed.  For dx the same holds of rounding x.)
 *   dy [rows][n_out] of `type`; dw_in, dw float [n_out][n_in] with rows ld_dw apart
 *   dw_in   NULL = zero; may be dw (rows of both at most PP_LAYER_MAX_LD_DW apart)
 *   db      float [n_out], or NULL = not wanted
 * With rows = 0, dw = dw_in and db = 0.
 */
int pp_linear_backward_weight(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *dy, int64_t ld_dy,
                              const void *x_codes, const void *x_scales, const float *dw_in, float *dw, int64_t ld_dw,
                              float *db, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PP_LAYER_H */
