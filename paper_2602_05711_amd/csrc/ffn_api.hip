// Host side of the entry points declared in include/omnimoe_ffn.h: argument checks, workspace carving and launches.
#include <hip/hip_runtime.h>

#include "../../include/omnimoe_ffn.h"
#include "checks.hpp"

using namespace omnimoe;

namespace {

omnimoe_status check_adapters(const omnimoe_adapters* a) {
  if (!a || a->n < 0 || a->rank < 8 || a->rank > 256 || a->rank % 8) return OMNIMOE_ERR_INVALID_ARG;
  return a->n > 8192 ? OMNIMOE_ERR_UNSUPPORTED : OMNIMOE_OK;
}

}  // namespace

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

omnimoe_status omnimoe_shared_mlp_adapters_workspace_size(const omnimoe_layer_desc* desc, int32_t d_ff,
                                                          const omnimoe_adapters* adapters, size_t* bytes) {
  if (!bytes || !valid_d_ff(d_ff)) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st || (st = check_adapters(adapters))) return st;
  *bytes = adapters_ws_bytes(s, d_ff, adapters->n, adapters->rank);
  return OMNIMOE_OK;
}

omnimoe_status omnimoe_shared_mlp_adapters(const omnimoe_layer_desc* desc, int32_t d_ff,
                                           const omnimoe_adapters* adapters, const void* x, const void* w_gu,
                                           const void* w_down, const int32_t* ids, const float* y_in, void* y,
                                           void* ws, size_t ws_bytes, void* stream) {
  if (!valid_d_ff(d_ff)) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  omnimoe_status st = check_desc(desc, &s);
  if (st || (st = check_adapters(adapters))) return st;
  if (s.T == 0) return OMNIMOE_OK;
  const omnimoe_adapters& a = *adapters;
  if ((st = check_ptrs({x, w_gu, w_down, ids, y, ws})) || (st = check_opt(y_in)) || (st = check_opt(a.scale))) return st;
  if (a.n && (st = check_ptrs({a.a_gu, a.b_gu, a.a_down, a.b_down}))) return st;
  if (ws_bytes < adapters_ws_bytes(s, d_ff, a.n, a.rank)) return OMNIMOE_ERR_WORKSPACE;
  const AdapterTables t{a.n, a.rank, a.a_gu, a.b_gu, a.a_down, a.b_down, a.scale};
  return hip_status(launch_adapters(s, d_ff, t, x, w_gu, w_down, ids, y_in, y, ws, (hipStream_t)stream));
}

}  // extern "C"
