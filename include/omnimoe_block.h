/*
 * omnimoe_block.h - the block around the layer and routed experts with matrices of their own (libomnimoe.so): the norms,
 * gate and residual scale that join a branch to the residual stream, matrix products of rows grouped by expert on
 * omnimoe_schedule's order, and the same products with 4-bit weights; with their gradients.
 *
 * Conventions as in omnimoe.h: device pointers owned by the caller, row-major, contiguous, 16-byte aligned; nothing is
 * allocated; every call is asynchronous on `stream`, checked on the host before anything is launched, and may run
 * beside calls on other streams with other workspaces; the workspace and all outputs must not overlap the inputs or
 * each other (but where a comment allows it), and the workspace's contents need not be initialised. `stream` belongs to
 * the calling thread's current device, which holds the tensors. Descriptors are checked whole. Results are the same on
 * every run. Unlike omnimoe.h's, inputs may hold infinities and NaN: they reach the rows that read them, and sums over
 * the rows, only.
 */
#ifndef OMNIMOE_BLOCK_H
#define OMNIMOE_BLOCK_H

#include "omnimoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Joins a branch to the residual stream and prepares the next branch's input. For each token, with norm(v) =
 * v / sqrt(mean(v^2) + eps) over its d values:
 *   x_out = x + scale * sigmoid(gate) * w_out * norm(y),   n = w_in * norm(x_out)
 *   x      [T, d]  dtype  the residual stream
 *   y      [T, d]  fp32   the branch's output (omnimoe_layer_forward's, with omnimoe_shared_mlp's added); NULL: x_out = x,
 *                         which is not written; gate, w_out, scale and x_out are then not used
 *   gate   [T, gate_width] dtype, gate_width 0, 1 (one for a token) or d; NULL with gate_width 0: factor 1
 *   w_out  [d] fp32, the weight of the norm behind the branch; NULL: y enters as it is
 *   scale  [d] fp32, the residual scale; NULL: 1
 *   w_in   [d] fp32, the weight of the norm before the next branch; NULL: n is not written (with y NULL: invalid)
 *   x_out  [T, d]  dtype out, may be x itself
 *   n      [T, d]  dtype out
 *   eps    1e-30 or more (squares that fp32 does not hold are then nothing beside it), finite
 * Of the descriptor T, d and dtype. Arithmetic is fp32; x_out and n are rounded once each, n from x_out before it is
 * rounded. Rows whose mean square is past fp32's largest value are normed as others. T = 0 is a no-op. */
omnimoe_status omnimoe_block_join(const omnimoe_layer_desc* desc, float eps, int32_t gate_width, const void* x,
                                  const float* y, const void* gate, const float* w_out, const float* scale,
                                  const float* w_in, void* x_out, void* n, void* stream);

/* Gradients of omnimoe_block_join for a loss L with dL/dx_out = dx_out (from what reads the stream later) and dL/dn = dn.
 *   x_out  [T, d]  dtype  omnimoe_block_join's x_out (with y NULL: its x)
 *   y, gate, w_out, scale, w_in   as there
 *   dx_out [T, d]  dtype, NULL: zeros (then w_in must be there);  dn [T, d] dtype, not used with w_in NULL
 *   dx     [T, d]  dtype out  dL/dx; may be dx_out or dn itself
 *   dy     [T, d]  fp32 out   dL/dy, as omnimoe_expert_backward and omnimoe_shared_mlp_backward take it
 *   dgate  [T, gate_width] dtype out
 *   dw_out, dscale, dw_in  [d] fp32 out, sums over the tokens
 * Outputs whose input is NULL (or with y NULL: not used) are not written and may be NULL. Without w_out dy does not depend on y.
 * The norms are formed again from
 * x_out and y. A row's sums are fp32: squares past its largest value are no matter, products of the row's gradients (w_in dn,
 * and those of w_out norm(y)) with x_out and norm(y) that are past it are. T = 0 writes zeros to those of the three sums that
 * are not NULL and uses nothing else. Workspace:
 * omnimoe_block_join_backward_workspace_size bytes. */
omnimoe_status omnimoe_block_join_backward_workspace_size(const omnimoe_layer_desc* desc, size_t* bytes);
omnimoe_status omnimoe_block_join_backward(const omnimoe_layer_desc* desc, float eps, int32_t gate_width,
                                           const void* x_out, const float* y, const void* gate, const float* w_out,
                                           const float* scale, const float* w_in, const void* dx_out, const void* dn,
                                           void* dx, float* dy, void* dgate, float* dw_out, float* dscale, float* dw_in,
                                           void* workspace, size_t workspace_bytes, void* stream);

/* Products of rows grouped by expert: experts that have a matrix each, run on omnimoe_schedule's order. Of the descriptor
 * T, n_rows * n_cols = N experts (at most 4096), H, K and dtype; M = T H K tasks (at most 2^31 - 1024; else
 * OMNIMOE_ERR_UNSUPPORTED).
 *   offsets [N + 1] int32  expert e's positions are offsets[e] .. offsets[e + 1] - 1 (omnimoe_schedule's dense_offsets, with
 *                          group_size 1): ascending, from 0 to M at most; an expert may have none. Positions from offsets[N]
 *                          on belong to nobody: they are not read and their outputs are left as they were. With N = 1 it
 *                          may be NULL: all M positions.
 *   perm    [M] int32      the task at each position; NULL where x_order and y_order are OMNIMOE_ORDER_POSITION. Used
 *                          otherwise, and a position whose entry is outside [0, M) then belongs to nobody. No task may
 *                          come twice where rows are written by task.
 * Rows of x and y lie by position (row p), by task (row perm[p]) or by token (row perm[p] / (H K); x only). */
enum { OMNIMOE_ORDER_POSITION = 0, OMNIMOE_ORDER_TASK = 1, OMNIMOE_ORDER_TOKEN = 2 };
typedef struct {
  int32_t n_in;    /* width of x's rows, 8 <= n_in <= 65536, n_in % 8 == 0 (4-bit weights: n_in % 32 == 0) */
  int32_t n_out;   /* width of y's rows, the same */
  int32_t swiglu;  /* 0: y = W x, W [n_out, n_in]. 1: y = silu(G x) (U x), W [2 n_out, n_in] being G's rows, then U's */
  int32_t x_order;
  int32_t y_order;
} omnimoe_product;

/* y = W_e x for every position of every expert e (or silu(G_e x) (U_e x), for use without gradients: a training step takes the
 * plain product of both halves and forms silu(g) u itself).
 *   x  [M, n_in], by token [T, n_in]   dtype
 *   w  [N, n_out, n_in], with swiglu [N, 2 n_out, n_in]  dtype; a matrix below 4 GiB, else OMNIMOE_ERR_UNSUPPORTED
 *   y  [M, n_out]  dtype out, rounded once from fp32 sums
 * T = 0 is a no-op. */
omnimoe_status omnimoe_grouped_product(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* x,
                                       const void* w, const int32_t* offsets, const int32_t* perm, void* y, void* stream);

/* Its gradients (swiglu 0) for dL/dy = dy [M, n_out] in dtype, which lies in y's order.
 *   dx  [M, n_in] dtype out   W_e^T dy, in x's order (by position or by task: a token's tasks have a row each)
 *   dw  [N, n_out, n_in] dtype out   sum over e's positions of dy x^T; zeros where e has none
 * T = 0 is a no-op for dx and writes zeros to dw (pointers to rows may then be NULL). Workspace of dw:
 * omnimoe_grouped_product_dw_workspace_size bytes (it may be 0, and the workspace NULL). */
omnimoe_status omnimoe_grouped_product_dx(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* dy,
                                          const void* w, const int32_t* offsets, const int32_t* perm, void* dx,
                                          void* stream);
omnimoe_status omnimoe_grouped_product_dw_workspace_size(const omnimoe_layer_desc* desc, const omnimoe_product* product,
                                                         size_t* bytes);
omnimoe_status omnimoe_grouped_product_dw(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* x,
                                          const void* dy, const int32_t* offsets, const int32_t* perm, void* dw,
                                          void* workspace, size_t workspace_bytes, void* stream);

/* Weights in 4 bits. Every row of w is cut into blocks of 32 values; a block is held as e2m1 codes (0, 0.5, 1, 1.5, 2, 3,
 * 4, 6, and a sign) times a power of two.
 *   w       [N, n_out, n_in], with swiglu [N, 2 n_out, n_in]  dtype
 *   codes   [N, .., n_in / 2]   uint8   value 2 i of a row in the low four bits of byte i, value 2 i + 1 in the high ones;
 *                                       a sign bit above the place in the list
 *   scales  [N, .., n_in / 32]  uint8   exponent + 127 of the block's power of two 2^s: the least s, -125 <= s <= 125, with
 *                                       max |w| <= 6 2^s
 * store: code = w 2^-s rounded to the nearest of the list, ties to the even place; magnitudes past 6 2^125 become that. A
 * block that holds a value which is not finite has scale byte 255, and all of its values are NaN.
 * load: w = code 2^s, exact in both types, for the scale bytes that store writes: 2 to 252, and 255.
 * Of the descriptor N and dtype, of the product n_in (n_in % 32 == 0), n_out and swiglu. */
omnimoe_status omnimoe_weights4_store(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* w,
                                      uint8_t* codes, uint8_t* scales, void* stream);
omnimoe_status omnimoe_weights4_load(const omnimoe_layer_desc* desc, const omnimoe_product* product,
                                     const uint8_t* codes, const uint8_t* scales, void* w, void* stream);

/* omnimoe_grouped_product with 4-bit weights, for a few rows an expert: every code is read once for up to sixteen rows and
 * is exact in the product. More rows go through the weights again for every sixteen. A prompt's many rows are faster through
 * omnimoe_grouped_product where omnimoe_weights4_load's result is kept (64 bf16 experts of 2048 x 2048 with SwiGLU, 4096 rows:
 * 126 us, here 140), and with a load each time from about 160 rows an expert on (8192 rows: 319 us, here 262). */
omnimoe_status omnimoe_grouped_product4(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* x,
                                        const uint8_t* codes, const uint8_t* scales, const int32_t* offsets,
                                        const int32_t* perm, void* y, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OMNIMOE_BLOCK_H */
