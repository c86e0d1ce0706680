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
 *   - Inputs and outputs must not overlap unless said otherwise.  A workspace serves one call at a
 *     time: calls that may run at once, on two streams or in two graphs, have one each.
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

/*
 * Root-mean-square norm of rows with the residual's addition, forward:
 *   s = x + res (x alone where res is NULL);  inv = 1 / sqrt(mean over the row of s^2 + eps);  y = s inv gain
 *   x, res, total, y  [rows][cols], all of `type`
 *   gain    float [cols], or NULL = 1
 *   eps     a normal positive float, at most 2^126
 *   total   s, or NULL = not wanted; may be res or x (same base and ld)
 *   y, y_codes/y_scales          out: y and y packed with PP_PACK_INT8 (as pp_linear_backward_weight reads it);
 *                                either may be NULL, not both
 *   total_codes/total_scales     out: s packed with PP_PACK_INT8 for pp_norm_backward, or both NULL
 *   inv     float [rows] for pp_norm_backward, or NULL
 * Results are made from s in 32 bits, each rounded once.  (The sum of a row's squares has to be a float.)
 */
int pp_norm_forward(int type, int64_t rows, int64_t cols, const void *x, int64_t ld_x, const void *res, int64_t ld_res,
                    const float *gain, float eps, void *total, int64_t ld_total, void *y, int64_t ld_y, void *y_codes,
                    void *y_scales, void *total_codes, void *total_scales, float *inv, void *stream);

/*
 * Its backward pass.  With z = s inv:
 *   dx = inv (gain dy - z mean over the row of (gain dy z)) + dtotal;   dgain = dgain_in + sum over the rows of dy z
 * (dx is the gradient of x and of res.)
 *   dy, dtotal, dx  [rows][cols], all of `type`; dtotal: the gradient that reaches s beside the norm, or NULL = none;
 *                   dx may be dy or dtotal (same base and ld)
 *   s      the matrix `total` of `type`, or total_codes/total_scales; one of the two, the other NULL
 *   inv    float [rows], as pp_norm_forward gave it
 *   dgain  float [cols], or NULL = not wanted; dgain_in NULL = zero; may be dgain
 * The workspace (256-byte aligned; not needed where dgain is NULL and a row has at most 16384 columns) need not be kept.
 * What so many rows need serves fewer.  With rows = 0, dgain = dgain_in.
 */
size_t pp_norm_workspace_bytes(int type, int64_t rows, int64_t cols);
int pp_norm_backward(int type, int64_t rows, int64_t cols, const void *dy, int64_t ld_dy, const void *total, int64_t ld_total,
                     const void *total_codes, const void *total_scales, const float *inv, const float *gain, const void *dtotal,
                     int64_t ld_dtotal, void *dx, int64_t ld_dx, const float *dgain_in, float *dgain, void *workspace,
                     size_t workspace_bytes, void *stream);

/*
 * Gated linear recurrence over the rows (tokens) of sequences that lie one behind the other, channel by channel:
 *   h_t = a_t h_(t-1) + (1 - a_t) v_t,   a_t = 1 / (1 + exp(-gate_t))
 * Sequence n has rows starts[n] .. starts[n+1] - 1 (none: an empty one); before its first token h is h0[n].
 *   gate, v, h       [rows][cols], all of `type`
 *   starts  int32 [seqs + 1], not falling, in 0 .. rows (what is not so is held to it); NULL = one sequence of all rows
 *           (seqs 1).  Rows before the first sequence and behind the last say nothing and are not written.
 *   h0      float [seqs][cols], or NULL = zero
 *   h_last  float [seqs][cols] out: h behind the last token (h0 for an empty sequence), or NULL = not wanted
 *   kept    float [pp_scan_kept_rows][cols] out: states for pp_scan_backward, or NULL = not wanted
 * States are held in 32 bits, and what 16 tokens do to one is added up by itself, so one that is kept for many tokens does not drift.
 * rows and cols: ceil(rows / 128) ceil(cols / 64) <= 2^24.
 * The workspaces (256-byte aligned) need not be kept; what so many rows need serves fewer.  pp_scan_kept_rows (host function;
 * -1 if a size or the type is out of range): both calls need the same type, rows and cols.
 */
#define PP_SCAN_FORWARD 0
#define PP_SCAN_BACKWARD 1
size_t pp_scan_workspace_bytes(int call, int type, int64_t rows, int64_t cols);
int64_t pp_scan_kept_rows(int type, int64_t rows, int64_t cols);
int pp_scan_forward(int type, int64_t rows, int64_t cols, const void *gate, int64_t ld_gate, const void *v, int64_t ld_v,
                    int64_t seqs, const int32_t *starts, const float *h0, void *h, int64_t ld_h, float *h_last, float *kept,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its backward pass.  With g_t = dh_t + a_(t+1) g_(t+1) within a sequence, and dh_last added to the last token's:
 *   dv = (1 - a) g;   dgate = a (1 - a) (h_(t-1) - v) g;   dh0 = a g of the first token (dh_last for an empty sequence)
 *   dh, gate, v, dgate, dv  [rows][cols], all of `type`; dgate, dv of rows in no sequence stay as they are
 *   h0, kept          as in pp_scan_forward (h is computed again from them in 32 bits, and not read)
 *   dh_last, dh0      float [seqs][cols]; NULL = zero, not wanted
 */
int pp_scan_backward(int type, int64_t rows, int64_t cols, const void *dh, int64_t ld_dh, const void *gate, int64_t ld_gate,
                     const void *v, int64_t ld_v, int64_t seqs, const int32_t *starts, const float *h0, const float *kept,
                     const float *dh_last, void *dgate, int64_t ld_dgate, void *dv, int64_t ld_dv, float *dh0, void *workspace,
                     size_t workspace_bytes, void *stream);

/*
 * One token of each of `rows` sequences:  h = a state[slots[r]] + (1 - a) v, which also is the slot's new state.
 *   gate, v, h   [rows][cols], all of `type`
 *   slots   int32 [rows], different from each other, or NULL = row r has slot r; a row whose slot is not in
 *           0 .. n_slots - 1 (padding) is left out, and its h stays as it is
 *   state   float [n_slots][cols], in and out
 */
int pp_scan_step(int type, int64_t rows, int64_t cols, const void *gate, int64_t ld_gate, const void *v, int64_t ld_v,
                 int64_t n_slots, const int32_t *slots, float *state, void *h, int64_t ld_h, void *stream);

/*
 * Log probabilities of rows of logits.  With z = logits / temperature and p = softmax(z) over a row:
 *   logp     float [rows] out: ln p of tokens[r], or NULL; 0 for a token < 0 (padding), NaN for one >= cols
 *   entropy  float [rows] out: -sum p ln p, or NULL
 *   norm     float [rows][2] out for pp_logprob_backward (8-byte aligned): the largest logit m and the sum of
 *            exp((logits - m) / temperature); or NULL
 *   top      0 .. PP_TOP_MAX: how many of the largest logits are wanted, largest first, equal ones by their column
 *   top_index int32 [rows][top], top_logp float [rows][top]  out: their columns and ln p
 *   logits   [rows][cols] of `type`;  tokens int32 [rows] (NULL only without logp);  2^-20 <= temperature <= 2^20
 * A logit of -infinity (a mask) has p = 0 and is no alternative: what is missing at the end of a list has index -1 and logp
 * -infinity.  In a row of nothing else logp is -infinity and the entropy 0.  A row that holds a NaN or +infinity gives NaN, and
 * index -1.  The workspace (256-byte aligned) need not be kept; what so many rows, or a larger top, needs serves fewer.
 */
#define PP_TOP_MAX 128
size_t pp_logprob_workspace_bytes(int type, int64_t rows, int64_t cols, int top);
int pp_logprob_forward(int type, int64_t rows, int64_t cols, const void *logits, int64_t ld_logits, float temperature,
                       const int32_t *tokens, float *logp, float *entropy, float *norm, int top, int32_t *top_index,
                       float *top_logp, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The gradient of logp and entropy (dlogp, dentropy float [rows]; NULL = zero; entropy is needed with dentropy alone):
 *   dlogits_j = (dlogp ([j = token] - p_j) - dentropy p_j (ln p_j + entropy)) / temperature
 * dlogits of `type`, may be logits (same base and ld).  Rows without a token take no dlogp, and one of a token >= cols is NaN where
 * dlogp is given; rows of nothing but -infinity have gradient 0.  A row with neither a token's dlogp nor a dentropy (NULL or 0) has
 * gradient 0 whatever it holds.
 */
int pp_logprob_backward(int type, int64_t rows, int64_t cols, const void *logits, int64_t ld_logits, float temperature,
                        const int32_t *tokens, const float *norm, const float *dlogp, const float *entropy, const float *dentropy,
                        void *dlogits, int64_t ld_dlogits, void *stream);

/*
 * Distillation: the divergence of p = softmax(logits / temperature) from a teacher of whom each row's `top` entries are known
 * (as pp_logprob_forward gives them), and its gradient, in one call.
 *   PP_DISTILL_TOP   top_value are logits (or log probabilities); q = softmax(top_value / temperature) over the list:
 *                    loss = weight sum q (ln q - ln p),                          dlogits_j = weight (p_j - q_j) / temperature
 *   PP_DISTILL_REST  top_value are log probabilities (at this temperature); q = exp(top_value), and all columns that are not
 *                    listed are one more outcome, of r = 1 - sum q (0 if that is below 2^-20) and p_rest:
 *                    loss = weight (sum q (ln q - ln p) + r (ln r - ln p_rest)), dlogits_j as above for what is listed, beside it
 *                    weight p_j (1 - r / p_rest) / temperature
 *   top_index int32 [rows][top], top_value float [rows][top]; 1 <= top <= PP_TOP_MAX.  An index outside 0 .. cols - 1 is none; a
 *             column listed twice has the sum of the two q.  A row with no q at all (PP_DISTILL_TOP) has loss and gradient 0.
 *   weight    float [rows], or NULL = 1.  A row of weight 0 (padding) has loss and gradient 0 whatever it holds.
 *   loss      float [rows] out
 *   dlogits   [rows][cols] of `type` out, or NULL = not wanted; may be logits (same base and ld)
 * In a row of nothing but -infinity the loss is infinite (0 if the list has no q) and the gradient 0; one that holds a NaN or
 * +infinity gives NaN.  Calls with a gradient that have 128 MiB of logits or more go another way through them: the gradient beside the list is
 * rounded otherwise, and p_rest - r is a difference in 32 bits.  The workspace (256-byte aligned) need not be kept; what so many rows, or a longer
 * list, needs serves fewer.
 */
#define PP_DISTILL_TOP 0
#define PP_DISTILL_REST 1
size_t pp_distill_workspace_bytes(int type, int64_t rows, int64_t cols, int top);
int pp_distill_loss(int kind, int type, int64_t rows, int64_t cols, const void *logits, int64_t ld_logits, float temperature, int top,
                    const int32_t *top_index, const float *top_value, const float *weight, float *loss, void *dlogits,
                    int64_t ld_dlogits, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PP_LAYER_H */
