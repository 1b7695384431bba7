// Host side of the entry points declared in include/omnimoe_block.h: argument checks and launches.
#include <hip/hip_runtime.h>

#include "../../include/omnimoe_block.h"
#include "checks.hpp"

using namespace omnimoe;

namespace {

omnimoe_status check_join(const omnimoe_layer_desc* desc, float eps, int32_t gate_width, const void* y, const void* w_in,
                          Shape* s) {
  const omnimoe_status st = check_desc(desc, s);
  if (st) return st;
  if (!(eps >= 1e-30f) || eps > 3.402823466e38f) return OMNIMOE_ERR_INVALID_ARG;
  if (gate_width != 0 && gate_width != 1 && gate_width != s->d) return OMNIMOE_ERR_INVALID_ARG;
  return y || w_in || s->T == 0 ? OMNIMOE_OK : OMNIMOE_ERR_INVALID_ARG;
}

constexpr int64_t kMostRows = kIntMax - 1023;  // (a tile past the last position still counts in 32 bits)

bool valid_width(int32_t n) { return n >= 8 && n <= kMaxFeatures && n % 8 == 0; }

omnimoe_status check_product(const omnimoe_layer_desc* desc, const omnimoe_product* product, Shape* s, ProductShape* q) {
  const omnimoe_status st = check_desc(desc, s);
  if (st) return st;
  if (!product || !valid_width(product->n_in) || !valid_width(product->n_out)) return OMNIMOE_ERR_INVALID_ARG;
  if (product->swiglu != 0 && product->swiglu != 1) return OMNIMOE_ERR_INVALID_ARG;
  if (product->x_order < OMNIMOE_ORDER_POSITION || product->x_order > OMNIMOE_ORDER_TOKEN ||
      product->y_order < OMNIMOE_ORDER_POSITION || product->y_order > OMNIMOE_ORDER_TASK)
    return OMNIMOE_ERR_INVALID_ARG;
  *q = {product->n_in, product->n_out, product->swiglu == 1, product->x_order, product->y_order};
  if (s->N > kMaxExperts || s->M > kMostRows) return OMNIMOE_ERR_UNSUPPORTED;
  const int64_t matrix = (int64_t)(q->swiglu ? 2 : 1) * q->n_out * q->n_in * (s->bf16 ? 2 : 4);
  return matrix >= (int64_t(1) << 32) ? OMNIMOE_ERR_UNSUPPORTED : OMNIMOE_OK;
}

// The schedule's arrays: which must be there, and perm as the kernels take it.
omnimoe_status check_rows(const Shape& s, const ProductShape& q, const int32_t* offsets, const int32_t** perm) {
  if (!offsets && s.N > 1) return OMNIMOE_ERR_INVALID_ARG;
  omnimoe_status st = check_opt(offsets);
  if (st) return st;
  if (q.x_order == OMNIMOE_ORDER_POSITION && q.y_order == OMNIMOE_ORDER_POSITION) {
    *perm = nullptr;
    return OMNIMOE_OK;
  }
  return check_ptrs({*perm});
}

omnimoe_status check_blocks(const ProductShape& q) { return q.n_in % 32 ? OMNIMOE_ERR_INVALID_ARG : OMNIMOE_OK; }

}  // namespace

extern "C" {

omnimoe_status omnimoe_block_join(const omnimoe_layer_desc* desc, float eps, int32_t gate_width, const void* x,
                                  const float* y, const void* gate, const float* w_out, const float* scale,
                                  const float* w_in, void* x_out, void* n, void* stream) {
  Shape s;
  omnimoe_status st = check_join(desc, eps, gate_width, y, w_in, &s);
  if (st) return st;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({x}))) return st;
  if (w_in && (st = check_ptrs({w_in, n}))) return st;
  if (y) {
    if ((st = check_ptrs({y, x_out})) || (st = check_opt(w_out)) || (st = check_opt(scale))) return st;
    if (gate_width && (st = check_ptrs({gate}))) return st;
  }
  return hip_status(launch_join(s.T, s.d, s.bf16, eps, gate_width, x, y, gate, w_out, scale, w_in, x_out, n,
                                (hipStream_t)stream));
}

omnimoe_status omnimoe_block_join_backward_workspace_size(const omnimoe_layer_desc* desc, size_t* bytes) {
  if (!bytes) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  const omnimoe_status st = check_desc(desc, &s);
  if (st) return st;
  *bytes = join_back_ws_bytes(s.T, s.d);
  return OMNIMOE_OK;
}

omnimoe_status omnimoe_block_join_backward(const omnimoe_layer_desc* desc, float eps, int32_t gate_width,
                                           const void* x_out, const float* y, const void* gate, const float* w_out,
                                           const float* scale, const float* w_in, const void* dx_out, const void* dn,
                                           void* dx, float* dy, void* dgate, float* dw_out, float* dscale, float* dw_in,
                                           void* ws, size_t ws_bytes, void* stream) {
  Shape s;
  omnimoe_status st = check_join(desc, eps, gate_width, y, w_in, &s);
  if (st) return st;
  if (s.T == 0) {  // (which inputs there are can not be told from their pointers)
    if ((st = check_opt(dw_out)) || (st = check_opt(dscale)) || (st = check_opt(dw_in))) return st;
    return hip_status(launch_join_back(0, s.d, s.bf16, eps, 0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                       nullptr, nullptr, nullptr, nullptr, dw_out, dscale, dw_in, nullptr,
                                       (hipStream_t)stream));
  }
  if (!dx_out && !w_in) return OMNIMOE_ERR_INVALID_ARG;
  if (w_in && (st = check_ptrs({w_in, dw_in}))) return st;
  if (y && w_out && (st = check_ptrs({w_out, dw_out}))) return st;
  if (y && scale && (st = check_ptrs({scale, dscale}))) return st;
  if ((st = check_ptrs({dx, ws})) || (st = check_opt(dx_out))) return st;
  if (w_in && (st = check_ptrs({x_out, dn}))) return st;
  if (y && (st = check_ptrs({y, dy}))) return st;
  if (y && gate_width && (st = check_ptrs({gate, dgate}))) return st;
  if (ws_bytes < join_back_ws_bytes(s.T, s.d)) return OMNIMOE_ERR_WORKSPACE;
  return hip_status(launch_join_back(s.T, s.d, s.bf16, eps, y ? gate_width : 0, x_out, y, gate, y ? w_out : nullptr,
                                     y ? scale : nullptr, w_in, dx_out, dn, dx, dy, dgate, y && w_out ? dw_out : nullptr,
                                     y && scale ? dscale : nullptr, w_in ? dw_in : nullptr, ws, (hipStream_t)stream));
}

omnimoe_status omnimoe_grouped_product(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* x,
                                       const void* w, const int32_t* offsets, const int32_t* perm, void* y,
                                       void* stream) {
  Shape s;
  ProductShape q;
  omnimoe_status st = check_product(desc, product, &s, &q);
  if (st) return st;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({x, w, y})) || (st = check_rows(s, q, offsets, &perm))) return st;
  return hip_status(launch_grouped_product(s, q, x, w, offsets, perm, y, (hipStream_t)stream));
}

omnimoe_status omnimoe_grouped_product_dx(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* dy,
                                          const void* w, const int32_t* offsets, const int32_t* perm, void* dx,
                                          void* stream) {
  Shape s;
  ProductShape q;
  omnimoe_status st = check_product(desc, product, &s, &q);
  if (st) return st;
  if (q.swiglu || q.x_order == OMNIMOE_ORDER_TOKEN) return OMNIMOE_ERR_INVALID_ARG;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({dy, w, dx})) || (st = check_rows(s, q, offsets, &perm))) return st;
  return hip_status(launch_grouped_dx(s, q, dy, w, offsets, perm, dx, (hipStream_t)stream));
}

omnimoe_status omnimoe_grouped_product_dw_workspace_size(const omnimoe_layer_desc* desc, const omnimoe_product* product,
                                                         size_t* bytes) {
  if (!bytes) return OMNIMOE_ERR_INVALID_ARG;
  Shape s;
  ProductShape q;
  const omnimoe_status st = check_product(desc, product, &s, &q);
  if (st) return st;
  if (q.swiglu) return OMNIMOE_ERR_INVALID_ARG;
  *bytes = grouped_dw_ws_bytes(s, q);
  return OMNIMOE_OK;
}

omnimoe_status omnimoe_grouped_product_dw(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* x,
                                          const void* dy, const int32_t* offsets, const int32_t* perm, void* dw, void* ws,
                                          size_t ws_bytes, void* stream) {
  Shape s;
  ProductShape q;
  omnimoe_status st = check_product(desc, product, &s, &q);
  if (st) return st;
  if (q.swiglu) return OMNIMOE_ERR_INVALID_ARG;
  if ((st = check_ptrs({dw}))) return st;
  if (s.T > 0) {
    if ((st = check_ptrs({x, dy})) || (st = check_rows(s, q, offsets, &perm))) return st;
    if (const size_t need = grouped_dw_ws_bytes(s, q)) {
      if ((st = check_ptrs({ws}))) return st;
      if (ws_bytes < need) return OMNIMOE_ERR_WORKSPACE;
    }
  } else {
    offsets = perm = nullptr;  // no positions
  }
  return hip_status(launch_grouped_dw(s, q, x, dy, offsets, perm, dw, ws, (hipStream_t)stream));
}

omnimoe_status omnimoe_weights4_store(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* w,
                                      uint8_t* codes, uint8_t* scales, void* stream) {
  Shape s;
  ProductShape q;
  omnimoe_status st = check_product(desc, product, &s, &q);
  if (st || (st = check_blocks(q)) || (st = check_ptrs({w, codes, scales}))) return st;
  return hip_status(launch_weights4_store(s, q, w, codes, scales, (hipStream_t)stream));
}

omnimoe_status omnimoe_weights4_load(const omnimoe_layer_desc* desc, const omnimoe_product* product,
                                     const uint8_t* codes, const uint8_t* scales, void* w, void* stream) {
  Shape s;
  ProductShape q;
  omnimoe_status st = check_product(desc, product, &s, &q);
  if (st || (st = check_blocks(q)) || (st = check_ptrs({codes, scales, w}))) return st;
  return hip_status(launch_weights4_load(s, q, codes, scales, w, (hipStream_t)stream));
}

omnimoe_status omnimoe_grouped_product4(const omnimoe_layer_desc* desc, const omnimoe_product* product, const void* x,
                                        const uint8_t* codes, const uint8_t* scales, const int32_t* offsets,
                                        const int32_t* perm, void* y, void* stream) {
  Shape s;
  ProductShape q;
  omnimoe_status st = check_product(desc, product, &s, &q);
  if (st || (st = check_blocks(q))) return st;
  if (s.T == 0) return OMNIMOE_OK;
  if ((st = check_ptrs({x, codes, scales, y})) || (st = check_rows(s, q, offsets, &perm))) return st;
  return hip_status(launch_grouped_product4(s, q, x, codes, scales, offsets, perm, y, (hipStream_t)stream));
}

}  // extern "C"
