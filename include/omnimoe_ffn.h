/*
 * omnimoe_ffn.h - the feed-forward layer around the routed branch (libomnimoe.so): the shared branch's training step
 * on 8-bit activation checkpoints, the shared branch with low-rank adapters, and the whole layer for a few tokens.
 *
 * Conventions as in omnimoe.h: device pointers owned by the caller, row-major, contiguous, 16-byte aligned; nothing is
 * allocated; every call is asynchronous on `stream`, checked on the host before anything is launched, and may run
 * beside calls on other streams with other workspaces; the workspace and all outputs must not overlap the inputs or
 * each other (but where a comment allows it), and the workspace's contents need not be initialised. `stream` belongs to
 * the calling thread's current device, which holds the tensors. Of the descriptor the calls here use T, d and dtype
 * unless stated otherwise; it is checked whole. Results are the same on every run.
 */
#ifndef OMNIMOE_FFN_H
#define OMNIMOE_FFN_H

#include "omnimoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activation checkpoint in 8 bits. Every row of x is cut into blocks of 32 values (the last one may be shorter); a
 * block is held as e4m3 codes (OCP: bias 7, largest 448) times a power of two.
 *   x       [T, d]            dtype
 *   codes   [T, d]            uint8
 *   scales  [T, ceil(d/32)]   uint8   exponent + 127 of the block's power of two 2^s: the least s >= -127 with
 *                                     max |x| <= 448 2^s
 * store: code = x 2^-s rounded to the nearest e4m3 value, ties to even (so within 2^-4 of the value, relative, where
 * |x| >= 2^(s-6), and within 2^(s-10) below). Values that are not finite are stored as NaN and take no part in the
 * block's maximum.
 * load: x = code 2^s in dtype, exact but where the type has no such small value; one past its largest finite value
 * (the rounding of a neighbour of that) becomes that. */
omnimoe_status omnimoe_checkpoint_store(const omnimoe_layer_desc* desc, const void* x, uint8_t* codes,
                                        uint8_t* scales, void* stream);
omnimoe_status omnimoe_checkpoint_load(const omnimoe_layer_desc* desc, const uint8_t* codes, const uint8_t* scales,
                                       void* x, void* stream);

/* Gradients of the shared branch (omnimoe_shared_mlp) for a loss L with dL/dy = dy, from the checkpoint of its input:
 * with x = the checkpoint's values, g = W_g x, u = W_u x (recomputed), a = silu(g) u, da = W_down^T dy,
 * dg = da u silu'(g), du = da silu(g):
 *   codes, scales             the checkpoint of x [T, d]
 *   w_gu     [2 d_ff, d], w_down [d, d_ff]   dtype, as in omnimoe_shared_mlp
 *   dy       [T, d]  fp32
 *   dx_in    [T, d]  fp32, may be NULL (zeros): the routed branch's share of dL/dx (omnimoe_expert_backward's with
 *                    omnimoe_route_backward's added)
 *   dx       [T, d]  dtype out   dx_in + W_g^T dg + W_u^T du, rounded once (fp32: may be dx_in itself)
 *   dw_gu    [2 d_ff, d] dtype out   sums over the tokens of dg x^T, then of du x^T
 *   dw_down  [d, d_ff]   dtype out   sum over the tokens of dy a^T
 * Sums are fp32 (matrix cores). bf16 layers round a, dg and du to bf16 between the products and take dy as the sum of two
 * bf16 values (2^-17 relative; an infinity in w_down or a can give NaN where the formula has an infinity). T = 0 writes
 * zeros to dw_gu and dw_down (the pointers to tokens and the workspace may then be NULL). d_ff as in omnimoe_shared_mlp.
 * Workspace: omnimoe_shared_mlp_backward_workspace_size bytes. */
omnimoe_status omnimoe_shared_mlp_backward_workspace_size(const omnimoe_layer_desc* desc, int32_t d_ff,
                                                          size_t* bytes);
omnimoe_status omnimoe_shared_mlp_backward(const omnimoe_layer_desc* desc, int32_t d_ff, const uint8_t* codes,
                                           const uint8_t* scales, const void* w_gu, const void* w_down,
                                           const float* dy, const float* dx_in, void* dx, void* dw_gu, void* dw_down,
                                           void* workspace, size_t workspace_bytes, void* stream);

/* The whole feed-forward layer (Eq. 7) for a decode step of a few tokens, in two kernels: omnimoe_layer_forward's routed
 * branch and, with d_ff > 0, omnimoe_shared_mlp's shared branch added to it.
 *   x, keys_row, keys_col, u, v   as in omnimoe_layer_forward (the whole descriptor counts; group_size is not used)
 *   w_gu, w_down                  as in omnimoe_shared_mlp; not used with d_ff = 0, and may then be NULL
 *   y [T, d] fp32 out;  idx_out, gates_out [T, H, K] out, as omnimoe_route's, may be NULL
 * The selection is exact on the fp32 logits, ties to the lower id. Routed sums are fp32 in (head, slot) order, each head's
 * by itself; the shared branch's hidden values enter the down projection unrounded, so that y has fp32's accuracy for
 * both types. Results agree with omnimoe_layer_forward's and omnimoe_shared_mlp's to the
 * rounding of their sums (and, for bf16 layers, of the hidden values there); logits summed in another order can put
 * near-ties the other way. T <= OMNIMOE_FEW_TOKENS and K <= 64, else OMNIMOE_ERR_UNSUPPORTED. T = 0 is a no-op.
 * When to take it: up to K = 32 it takes less time than those two calls (than the first alone with d_ff = 0). For K > 40, and
 * where a half has more than 64 but fewer than 4 K sub-keys, its selection goes one pick at a time; then, on grids below
 * 1024 x 1024, the two calls take less time for one token, and the first alone does with d_ff = 0 (320 x 320, K = 64, one
 * head: 39 instead of 53 us, without a shared branch 31).
 * Workspace: omnimoe_layer_few_workspace_size bytes. */
#define OMNIMOE_FEW_TOKENS 16
omnimoe_status omnimoe_layer_few_workspace_size(const omnimoe_layer_desc* desc, int32_t d_ff, size_t* bytes);
omnimoe_status omnimoe_layer_forward_few(const omnimoe_layer_desc* desc, int32_t d_ff, const void* x,
                                         const void* keys_row, const void* keys_col, const void* u, const void* v,
                                         const void* w_gu, const void* w_down, float* y, int32_t* idx_out,
                                         float* gates_out, void* workspace, size_t workspace_bytes, void* stream);

/* Low-rank adapters of the shared branch's projections, side by side in tables of n slots. All of a table's slots have the
 * same rank (a smaller one is filled up with zeros). Only slots that a token names are read.
 *   n       slots, 0 <= n <= 8192 (else OMNIMOE_ERR_UNSUPPORTED); with n = 0 the tables may be NULL
 *   rank    8 <= rank <= 256, rank % 8 == 0
 *   a_gu    [n, 2 rank, d]      dtype   the gate projection's A, then the up projection's
 *   b_gu    [n, 2 d_ff, rank]   dtype   rows as w_gu's: the gate rows' B, then the up rows'
 *   a_down  [n, rank, d_ff]     dtype
 *   b_down  [n, d, rank]        dtype
 *   scale   [n] fp32, may be NULL (ones) */
typedef struct {
  int32_t n;
  int32_t rank;
  const void* a_gu;
  const void* b_gu;
  const void* a_down;
  const void* b_down;
  const float* scale;
} omnimoe_adapters;

/* The shared branch of a batch whose tokens belong to requests with adapters of their own. With e = ids[t]:
 *   g = W_g x + scale_e B_gate (A_gate x),  u = W_u x + scale_e B_up (A_up x),  a = silu(g) u,
 *   y = y_in + W_down a + scale_e B_down (A_down a)
 *   x [T, d], w_gu [2 d_ff, d], w_down [d, d_ff]   dtype, as in omnimoe_shared_mlp
 *   ids   [T] int32   the token's slot; a value outside [0, n): no adapter
 *   y_in  [T, d] fp32, may be NULL (zeros): e.g. omnimoe_layer_forward's y
 *   y     [T, d] dtype out, rounded once (fp32 layers: may be y_in itself)
 * Tokens of any adapters may come in any order; a token's result does not depend on the others in the batch but for the
 * rounding of sums, whose order differs between calls of up to 16, up to 64 and more tokens, and no value of another
 * slot enters it. Sums are fp32; bf16 layers round a (as omnimoe_shared_mlp does) and, from 65 tokens on, the rank-wide
 * values to bf16 for the matrix cores. T = 0 is a no-op. Workspace: omnimoe_shared_mlp_adapters_workspace_size bytes
 * (the tables' pointers and scale do not count there). */
omnimoe_status omnimoe_shared_mlp_adapters_workspace_size(const omnimoe_layer_desc* desc, int32_t d_ff,
                                                          const omnimoe_adapters* adapters, size_t* bytes);
omnimoe_status omnimoe_shared_mlp_adapters(const omnimoe_layer_desc* desc, int32_t d_ff,
                                           const omnimoe_adapters* adapters, const void* x, const void* w_gu,
                                           const void* w_down, const int32_t* ids, const float* y_in, void* y,
                                           void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OMNIMOE_FFN_H */
