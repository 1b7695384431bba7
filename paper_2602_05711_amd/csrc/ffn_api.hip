// Host side of the entry points declared in include/omnimoe_ffn.h: argument checks, workspace carving and launches.
#include <hip/hip_runtime.h>

#include "../../include/omnimoe_ffn.h"
#include "checks.hpp"

using namespace omnimoe;

extern "C" {

omnimoe_status omnimoe_checkpoint_store(const omnimoe_layer_desc* desc, const void* x, uint8_t* codes,
                                        uint8_t* scales, void* stream) {
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({x, codes, scales}))) return st;
  return hip_status(launch_checkpoint_store(s.T, s.d, s.bf16, x, codes, scales, (hipStream_t)stream));
}

omnimoe_status omnimoe_checkpoint_load(const omnimoe_layer_desc* desc, const uint8_t* codes, const uint8_t* scales,
                                       void* x, void* stream) {
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({codes, scales, x}))) return st;
  return hip_status(launch_checkpoint_load(s.T, s.d, s.bf16, codes, scales, x, (hipStream_t)stream));
}

omnimoe_status omnimoe_shared_mlp_backward_workspace_size(const omnimoe_layer_desc* desc, int32_t d_ff,
                                                          size_t* bytes) {
  if (!bytes || !valid_d_ff(d_ff)) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  *bytes = shared_backward_ws_bytes(s, d_ff);
  return OMNIMOE_OK;
}

omnimoe_status omnimoe_shared_mlp_backward(const omnimoe_layer_desc* desc, int32_t d_ff, const uint8_t* codes,
                                           const uint8_t* scales, const void* w_gu, const void* w_down,
                                           const float* dy, const float* dx_in, void* dx, void* dw_gu, void* dw_down,
                                           void* ws, size_t ws_bytes, void* stream) {
  if (!valid_d_ff(d_ff)) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  if ((st = check_ptrs({w_gu, w_down, dw_gu, dw_down}))) return st;
  if (s.T > 0) {
    if ((st = check_ptrs({codes, scales, dy, dx, ws})) || (st = check_opt(dx_in))) return st;
    if (ws_bytes < shared_backward_ws_bytes(s, d_ff)) return OMNIMOE_ERR_WORKSPACE;
  }
  return hip_status(launch_shared_backward(s, d_ff, codes, scales, w_gu, w_down, dy, dx_in, dx, dw_gu, dw_down, ws,
                                           (hipStream_t)stream));
}

omnimoe_status omnimoe_layer_few_workspace_size(const omnimoe_layer_desc* desc, int32_t d_ff, size_t* bytes) {
  if (!bytes || (d_ff != 0 && !valid_d_ff(d_ff))) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  if (!few_fits(s)) return OMNIMOE_ERR_UNSUPPORTED;
  *bytes = few_ws_bytes(s, d_ff);
  return OMNIMOE_OK;
}

omnimoe_status omnimoe_layer_forward_few(const omnimoe_layer_desc* desc, int32_t d_ff, const void* x,
                                         const void* keys_row, const void* keys_col, const void* u, const void* v,
                                         const void* w_gu, const void* w_down, float* y, int32_t* idx_out,
                                         float* gates_out, void* ws, size_t ws_bytes, void* stream) {
  if (d_ff != 0 && !valid_d_ff(d_ff)) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  if (!few_fits(s)) return OMNIMOE_ERR_UNSUPPORTED;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({x, keys_row, keys_col, u, v, y, ws}))) return st;
  if (d_ff && (st = check_ptrs({w_gu, w_down}))) return st;
  if ((st = check_opt(idx_out)) || (st = check_opt(gates_out))) return st;
  if (ws_bytes < few_ws_bytes(s, d_ff)) return OMNIMOE_ERR_WORKSPACE;
  return hip_status(launch_few(s, d_ff, x, keys_row, keys_col, u, v, w_gu, w_down, y, idx_out, gates_out, ws,
                               (hipStream_t)stream));
}

}  // extern "C"
