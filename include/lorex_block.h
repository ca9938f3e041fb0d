/*
 * lorex_block.h -- the operators around the expert layer, and the experts in
 * microscaled 4-bit floating point.
 *
 *   block norms    the norms before and after a block, fused with the block's
 *                  gate, its residual scale and the sum over a token's experts
 *   balance loss   the router's load-balance loss, the tokens per expert, and
 *                  the gradient of the logits
 *   dropout        of the block's output inside these norms, from a
 *                  counter-based generator: the mask is never stored
 *   4-bit values   rounding to OCP MXFP4 (blocks of 32 values with one
 *                  power-of-two scale), reading back, and products of two
 *                  4-bit operands, one weight matrix per group of rows
 *   few tokens     a whole layer of experts in 4 bits for decoding, in two
 *                  launches
 *   8-bit values   rounding to OCP MXFP8 (e4m3), also straight from the norms,
 *                  reading back, and products of 8-bit activations and 4-bit
 *                  weights with a bias, an activation and a residual
 *
 * The conventions of lorex.h hold: device pointers to dense row-major
 * caller-owned memory, asynchronous on `stream`, nothing allocated, no
 * pointer kept, argument errors returned before anything is enqueued
 * (lx_last_error), workspaces that need no initialisation. Memory and `stream`
 * belong to the GPU that is current at the call. Every call may be
 * captured into a HIP graph. Results do not change from run to run: no sum
 * depends on the order in which workgroups run.
 */
#ifndef LOREX_BLOCK_H
#define LOREX_BLOCK_H

#include "lorex.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------ block norms
 * Around a block (attention, or the MoE layer of lorex.h) a model keeps a
 * residual stream h. With rms(v) = (mean_c v_c^2 + eps)^(-1/2) per token:
 *
 *   y      the block's output row, or with slot_row / slot_weights the sum
 *          over the token's k slots of slot_weights[t][j] Y[slot_row[t][j]]
 *   v      = y rms(y) w_post          (w_post NULL: v = y)
 *   h_out  = residual_scale h + gate_t scale_c v     (gate, scale NULL: 1)
 *   x      = h_out rms(h_out) w_pre   (the next block's input)
 *
 * Everything is computed in fp32 from the values as stored and rounded once
 * on output: x comes from the unrounded h_out. */
typedef struct lx_norm_layer {
  int32_t d;                 /* channels: a multiple of 8, at most LX_NORM_MAX_D */
  lx_dtype h_dtype;          /* of h, h_out and their gradients */
  lx_dtype y_dtype;          /* of y (Y) and dy */
  lx_dtype x_dtype;          /* of x and dx */
  lx_dtype w_dtype;          /* of w_pre, w_post and scale */
  float residual_scale;      /* factor of h */
  float eps;                 /* >= 0, added to the mean square */
  const void* w_pre;         /* [d] or NULL: no x is computed */
  const void* w_post;        /* [d] or NULL: the block's output is not normalised */
  const void* scale;         /* [d] or NULL */
  const float* gate;         /* [T] fp32 or NULL */
} lx_norm_layer;

#define LX_NORM_MAX_D 32768

/* h [T][d]; y NULL (no block: x = h rms(h) w_pre, h_out must be NULL, and
 * w_post, scale and gate are not read), [T][d], or, with slot_row [T][k]
 * int32 and slot_weights [T][k] fp32 (both or neither), the rows Y
 * [y_rows][d]: a slot whose row is outside [0, y_rows) adds nothing, a token
 * without any slot gets y = 0. Without slots y_rows and k are ignored. k in 1
 * .. LX_MAX_K. h_out [T][d] (may be h itself), x [T][d] (given exactly when
 * w_pre is). T = 0 does nothing. All but slots and gate 16-byte aligned. */
lx_status lx_block_norm(const lx_norm_layer* layer, int32_t T, const void* h, const void* y, int32_t y_rows,
                        int32_t k, const int32_t* slot_row, const float* slot_weights, void* h_out, void* x,
                        void* stream);

/* The gradients of lx_block_norm (without slots), from its inputs and from
 * h_out as it was stored (without w_pre not read): dx is the gradient of x
 * (NULL exactly when w_pre is), dh_out the gradient of h_out from elsewhere
 * (NULL: zero). Outputs: dh [T][d]; dy [T][d] (given exactly when y is); fp32
 * dgate [T], dw_pre [d], dw_post [d], dscale [d], each given exactly when its
 * input takes part. Without y (no block) h_out is the stream h itself and dh
 * its gradient. dh may be dh_out. T = 0 writes zeros to the gradients of the weights.
 * workspace 256-byte aligned, lx_block_norm_backward_workspace_bytes bytes. */
size_t lx_block_norm_backward_workspace_bytes(int32_t T, int32_t d);
lx_status lx_block_norm_backward(const lx_norm_layer* layer, int32_t T, const void* h_out, const void* y,
                                 const void* dx, const void* dh_out, void* dh, void* dy, float* dgate,
                                 float* dw_pre, float* dw_post, float* dscale, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------ dropout
 * The block norms with the (normalised) block's output dropped out before gate
 * and scale:
 *
 *   h_out  = residual_scale h + gate_t scale_c drop(v)_tc
 *   drop(v)_tc = v_tc / (1 - q) if u_tc >= 65536 q, else 0 (and scale_c drop(v)_tc
 *                too, whatever y_tc, w_post_c and scale_c hold)
 *
 * with q = p rounded to a multiple of 2^-16, 0 <= q < 1 (p from 1 - 2^-17 on is
 * refused), and 16 random bits u_tc from Philox4x32 of ten rounds: key = the
 * seed (low word first), counter = (c / 8, t, offset low, offset high); u_tc is
 * half c % 2 (0: the low one) of word (c % 8) / 2. rng: the seed and the offset,
 * two 64-bit integers on the device, 8-byte aligned, read when the kernels run: a
 * captured graph draws anew where the program moves the offset on between
 * replays. Every (layer, step, rank) takes an offset or a seed of its own; the
 * backward takes what the forward took and forms the mask again. p = 0 is the
 * plain norm, rng is not read then. */
typedef struct lx_dropout {
  float p;
  const int64_t* rng;        /* [2]: seed, offset */
} lx_dropout;

/* lx_block_norm without slots, lx_block_norm_backward; y must be given. */
lx_status lx_block_norm_dropout(const lx_norm_layer* layer, const lx_dropout* dropout, int32_t T, const void* h,
                                const void* y, void* h_out, void* x, void* stream);
lx_status lx_block_norm_dropout_backward(const lx_norm_layer* layer, const lx_dropout* dropout, int32_t T,
                                         const void* h_out, const void* y, const void* dx, const void* dh_out, void* dh,
                                         void* dy, float* dgate, float* dw_pre, float* dw_post, float* dscale,
                                         void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------ balance loss
 * lx_route_topk that leaves its logits [T][E] (fp32, 16-byte aligned) too: the
 * sums that ids and weights, which are those of lx_route_topk bit for bit, were
 * chosen and formed from, for the loss below. The other arguments, the
 * workspace among them, as there. */
lx_status lx_route_topk_logits(const void* x, const void* w_r, lx_dtype dtype, int32_t T, int32_t d, int32_t E,
                               int32_t k, int32_t* topk_ids, float* topk_weights, float* logits, void* workspace,
                               size_t workspace_bytes, void* stream);

/* For router logits [T][E] (fp32 or bf16) and the chosen experts topk_ids
 * [T][k] (as lx_route_topk writes them), over the N tokens whose mask byte is
 * not zero (mask NULL: all T):
 *
 *   p      = softmax(logits[t]);  counts[e] = slots of those tokens on e
 *   f_e    = counts[e] / (k N);   prob[e]   = (1 / N) sum_t p_te
 *   loss   = coef E sum_e f_e prob[e]        (coef for a balanced router)
 *   dlogits_te = dloss coef E / N p_te (f_e - sum_j f_j p_tj)
 *
 * ids outside [0, E) are not counted; a repeated id counts each time. A
 * logit of -inf is an expert that is switched off (p = 0, gradient 0); a row
 * of only -inf has p = 0 everywhere. A masked token's logits and ids are not
 * looked at and its gradient is 0; N = 0 gives 0 everywhere. NaN spreads.
 *
 * loss [1], prob [E] fp32, counts [E], n_tokens [1] int32, all written. E in
 * 1 .. 1024 (LX_ERR_UNSUPPORTED), k in 1 .. LX_MAX_K, T * k < 2^31. The
 * backward takes counts and n_tokens as the forward wrote them, or summed
 * over micro-batches or ranks; dloss is a device fp32 scalar (NULL: 1).
 * logits and dlogits 16-byte aligned; dlogits may be logits. */
size_t lx_balance_loss_workspace_bytes(int32_t T, int32_t E);
lx_status lx_balance_loss(const void* logits, lx_dtype dtype, int32_t T, int32_t E, const int32_t* topk_ids,
                          int32_t k, const uint8_t* mask, float coef, float* loss, int32_t* counts, float* prob,
                          int32_t* n_tokens, void* workspace, size_t workspace_bytes, void* stream);
lx_status lx_balance_loss_backward(const void* logits, lx_dtype dtype, int32_t T, int32_t E, int32_t k,
                                   const uint8_t* mask, const int32_t* counts, const int32_t* n_tokens, float coef,
                                   const float* dloss, void* dlogits, void* stream);

/* ------------------------------------------------------------ 4-bit values
 * OCP Microscaling MXFP4: 32 consecutive values share the scale 2^(s - 127)
 * (s an E8M0 byte, 255 = NaN) and are e2m1 codes: sign, then 0, 0.5, 1, 1.5,
 * 2, 3, 4, 6. A row of K values (K a multiple of 8) is padded with zeros to
 * Kp = LX_MX4_KP(K); its codes are Kp / 2 bytes (value 2i in the low half of
 * byte i), its scales Kp / 32 bytes. Rows follow each other without gaps. */
#define LX_MX4_KP(K) (((K) + 127) / 128 * 128)

/* What is rounded: the values themselves, or silu(g) u of rows [g (K) | u
 * (K)], the gate and up projections of a SwiGLU expert. */
typedef enum lx_mx4_act { LX_MX4_NONE = 0, LX_MX4_SWIGLU = 1 } lx_mx4_act;

/* x [rows][K] (LX_MX4_SWIGLU: [rows][2K]) -> codes [rows][Kp / 2], scales
 * [rows][Kp / 32], padding included. The scale's exponent is floor(log2 of the
 * block's largest magnitude) - 2, at least -127; values are rounded to the
 * nearest code, ties to even, and past 6 to 6. A block that holds an infinity
 * or a NaN gets the scale NaN and codes 0. x and codes 16-byte, scales 4-byte
 * aligned. */
lx_status lx_mx4_quantize(const void* x, lx_dtype dtype, int64_t rows, int32_t K, lx_mx4_act act, void* codes,
                          void* scales, void* stream);

/* codes, scales -> out [rows][K]; exact in both types (from 2^128 on infinite). */
lx_status lx_mx4_dequantize(const void* codes, const void* scales, int64_t rows, int32_t K, void* out,
                            lx_dtype dtype, void* stream);

/* out[m][n] = sum_c A[row(m)][c] B[g][n][c] in fp32, for the rows m of group g.
 * A: codes and scales of a_rows rows; row(m) = row_map[m], or m (row_map NULL,
 * a_rows >= M). B: G matrices of N rows. Rows offsets[g] .. offsets[g + 1] - 1
 * belong to group g (offsets [G + 1] int32 in ascending order, device; NULL:
 * G = 1 and all M rows); M is the most rows there can be: rows from offsets[G]
 * on are not written. Offsets outside [0, M] are clamped to it, and a row_map
 * entry outside [0, a_rows) gives a row of zeros, whatever the weights hold.
 * out [M][N] fp32 or bf16. K a multiple of 8, M and N at most 2^31 -
 * 256, M * N < 2^40, G in 1 .. LX_MAX_NODES. A, B and out 16-byte, their scales, row_map and
 * offsets 4-byte aligned; workspace 256-byte aligned,
 * lx_mx4_gemm_workspace_bytes bytes (NULL where that is 0).
 * The order in which a sum is formed depends on M, N, K, G and on whether A's
 * codes reach 2^32 bytes (or a_rows is 0): from there on the kernel of few rows
 * runs, which reads a group's weights once per 16 rows; rows that are gathered
 * from that far are better copied together first. */
size_t lx_mx4_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t G);
lx_status lx_mx4_gemm(const void* a, const void* a_scales, int32_t a_rows, const int32_t* row_map, const void* b,
                      const void* b_scales, const int32_t* offsets, int32_t G, int32_t M, int32_t N, int32_t K,
                      void* out, lx_dtype out_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------ few tokens
 * A layer of experts in 4 bits for up to LX_MOE_FEW_MAX_T tokens, in two launches:
 *
 *   out[t] = sum_j weights[t][j] down_e (silu(gate_e x_t) * (up_e x_t)),  e = ids[t][j]
 *
 * x [T][d] (fp32 or bf16) is not rounded; ids [T][k] int32 and weights [T][k] fp32
 * as lx_route_topk writes them: a slot whose id is outside [0, E) adds nothing,
 * a token may name an expert more than once, a token without any slot gets
 * zeros. gate_up: codes and scales of E x [2f][d] (gate rows first), down: of E
 * x [d][f]. Only the chosen experts' weights are read, each once per 16 of its
 * tokens; a NaN scale or an infinite activation reaches the tokens that it is
 * multiplied for only. Weights below 2^-126 under a block's scale may count as 0.
 * Sums are formed in fp32, and the activations between the two products keep its
 * 24 bits. out [T][d]. d and f multiples of 8, at most 2^20, E in 1 .. LX_MAX_NODES, k in 1 ..
 * LX_MAX_K (LX_ERR_UNSUPPORTED; T over the most as well). All 16-byte aligned but
 * ids, weights and scales (4); workspace 256-byte aligned, as many bytes as the
 * function before says. */
#define LX_MOE_FEW_MAX_T 64
size_t lx_mx4_moe_few_workspace_bytes(int32_t T, int32_t k, int32_t E, int32_t d, int32_t f);
lx_status lx_mx4_moe_few(const void* x, lx_dtype x_dtype, int32_t T, int32_t d, const int32_t* topk_ids,
                         const float* topk_weights, int32_t k, int32_t E, int32_t f, const void* gate_up,
                         const void* gate_up_scales, const void* down, const void* down_scales, void* out,
                         lx_dtype out_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------ 8-bit values
 * OCP Microscaling MXFP8: 32 consecutive values share the scale 2^(s - 127) (s an
 * E8M0 byte, 255 = NaN) and are e4m3 codes. A row of K values (K a multiple of 8)
 * is padded with zeros to Kp = LX_MX8_KP(K); its codes are Kp bytes, its scales
 * Kp / 32. Rows follow each other without gaps. */
#define LX_MX8_KP(K) (((K) + 127) / 128 * 128)

/* x [rows][K] (LX_MX4_SWIGLU: [rows][2K]) -> codes [rows][Kp], scales
 * [rows][Kp / 32], padding included. The scale is the smallest for which the
 * block's largest magnitude is at most 448 scales, at least 2^-127: no value
 * saturates. Values are rounded to the nearest code, ties to even. A block that
 * holds an infinity or a NaN gets the scale NaN and codes 0. x 16-byte, codes
 * 16-byte, scales 4-byte aligned. */
lx_status lx_mx8_quantize(const void* x, lx_dtype dtype, int64_t rows, int32_t K, lx_mx4_act act, void* codes,
                          void* scales, void* stream);

/* codes, scales -> out [rows][K]: exact in both types (but for infinities from
 * 2^128 on, and in bf16 for values below its smallest, 2^-133). */
lx_status lx_mx8_dequantize(const void* codes, const void* scales, int64_t rows, int32_t K, void* out,
                            lx_dtype dtype, void* stream);

/* Products per group of rows like lx_mx4_gemm, of 8-bit activations and 4-bit
 * weights, with what follows a projection:
 *
 *   z[m][n]   = sum_c A[row(m)][c] B[g][n][c] + bias[g][n]
 *   out[m][n] = act(z[m][n]) + residual[m][n]
 *
 * LX_ACT_SWIGLU: B's N rows are N / 2 gate rows, then N / 2 up rows, and out [M][N
 * / 2] = silu(z[m][n]) z[m][N / 2 + n] + residual[m][n]; GELU is z Phi(z). (silu here is by
 * the exponential and reciprocal instructions, in lx_mx8_quantize by expf and a division: a
 * value next to the border of two codes may get either.) A: codes [a_rows][LX_MX8_KP(K)] and
 * scales; B: as in lx_mx4_gemm; row_map, offsets, G, M,
 * rows of no group and map entries out of range (a product of 0 then, bias,
 * activation and residual as for any other row) as there. bias [G][N], residual
 * [M][columns], fp32 or bf16 each, aligned to their type; epilogue NULL: neither,
 * and no activation. Everything after the product is computed in fp32 and rounded
 * once. out [M][columns] fp32 or bf16 (out_scales NULL), or 8-bit values with rows of
 * `columns` (a multiple of 8) as lx_mx8_quantize rounds them: codes in out, scales
 * in out_scales, padding included; out_dtype is not looked at then. residual may
 * be out where their types agree.
 * K a multiple of 8, at most 2^24, M and N at most 2^31 - 256, M * N < 2^40, G in 1 ..
 * LX_MAX_NODES. A, B and out 16-byte, scales, row_map and offsets 4-byte aligned;
 * workspace 256-byte aligned, lx_mx8_gemm_workspace_bytes bytes (NULL where that is
 * 0). Products are exact in fp32, whatever the result's type. The order in which a sum
 * is formed depends on the sizes, G and act, not on the values or the result's type, and
 * for more than a few rows on whether A's codes or a group's weights reach 2^32 bytes (or
 * a_rows is 0): from there on the kernels of few rows run, which read a group's weights
 * once per 16 rows; rows that are gathered from that far are better copied together first. */
typedef enum lx_act { LX_ACT_NONE = 0, LX_ACT_SILU = 1, LX_ACT_GELU = 2, LX_ACT_SWIGLU = 3 } lx_act;
typedef struct lx_epilogue {
  lx_act act;
  lx_dtype bias_dtype;
  lx_dtype residual_dtype;
  const void* bias;          /* or NULL */
  const void* residual;      /* or NULL */
} lx_epilogue;
size_t lx_mx8_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t G, lx_act act);
lx_status lx_mx8_gemm(const void* a, const void* a_scales, int32_t a_rows, const int32_t* row_map, const void* b,
                      const void* b_scales, const int32_t* offsets, int32_t G, int32_t M, int32_t N, int32_t K,
                      const lx_epilogue* epilogue, void* out, lx_dtype out_dtype, void* out_scales, void* workspace,
                      size_t workspace_bytes, void* stream);

/* lx_block_norm whose x is rounded to 8 bits as lx_mx8_quantize rounds the
 * unrounded fp32 x: codes [T][LX_MX8_KP(d)] (16-byte aligned) and scales
 * [T][LX_MX8_KP(d) / 32] (4-byte aligned), padding included; both are given, as
 * is w_pre. x NULL, or [T][d] of layer.x_dtype: it is written too (for a router).
 * Its gradients are
 * lx_block_norm_backward's, from the gradient of the values (the rounding passes
 * it on). */
lx_status lx_block_norm_mx8(const lx_norm_layer* layer, int32_t T, const void* h, const void* y, int32_t y_rows,
                            int32_t k, const int32_t* slot_row, const float* slot_weights, void* h_out, void* x,
                            void* x_codes, void* x_scales, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LOREX_BLOCK_H */
