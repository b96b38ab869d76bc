// Host-side argument checks and sizes shared by the C-ABI sources.
#pragma once

#include <hip/hip_runtime.h>

#include <cstring>

#include "kvg.h"
#include "kvg_device.h"

namespace kvg {
namespace host {

constexpr size_t kAlign = 256;

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline size_t elem_bytes(const kvg_cache* c) { return c->dtype == KVG_BF16 ? 2 : c->dtype == KVG_FP8_E4M3 ? 1 : 4; }

inline int check_cache(const kvg_cache* c) {
  if (c == nullptr || c->k_pool == nullptr || c->v_pool == nullptr) return KVG_E_INVAL;
  if (c->dtype != KVG_F32 && c->dtype != KVG_BF16 && c->dtype != KVG_FP8_E4M3) return KVG_E_DTYPE;
  if (c->n_layers <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_pages <= 0) return KVG_E_SHAPE;
  if (c->n_pages > INT32_MAX) return KVG_E_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return KVG_E_SHAPE;
  if (c->page_size != kPage) return KVG_E_SHAPE;
  if (c->n_q_heads % c->n_kv_heads != 0) return KVG_E_SHAPE;
  const int g = c->n_q_heads / c->n_kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 8) return KVG_E_SHAPE;
  if (c->layer_window != nullptr)
    for (int l = 0; l < c->n_layers; ++l)
      if (c->layer_window[l] < 0) return KVG_E_INVAL;
  return KVG_OK;
}

// Windows of layers [layer0, layer0 + n_layers) as a launch carries them (all zero when none
// is windowed); KVG_E_SHAPE when a windowed call spans more layers than a launch carries.
inline int fill_windows(const kvg_cache* c, int32_t layer0, int32_t n_layers, int32_t* dst) {
  std::memset(dst, 0, sizeof(int32_t) * kvg::kMaxWindowLayers);
  if (c->layer_window == nullptr) return KVG_OK;
  bool any = false;
  for (int l = 0; l < n_layers; ++l) any = any || c->layer_window[layer0 + l] != 0;
  if (!any) return KVG_OK;
  if (n_layers > kvg::kMaxWindowLayers) return KVG_E_SHAPE;
  for (int l = 0; l < n_layers; ++l) dst[l] = c->layer_window[layer0 + l];
  return KVG_OK;
}

inline int check_layers(const kvg_cache* c, int32_t layer0, int32_t n_layers) {
  if (layer0 < 0 || n_layers <= 0 || layer0 + (int64_t)n_layers > c->n_layers) return KVG_E_SHAPE;
  return KVG_OK;
}

inline int64_t layer_elems(const kvg_cache* c) {
  return c->n_pages * c->n_kv_heads * (int64_t)c->page_size * c->head_dim;
}

inline int hip_status(hipError_t e) { return e == hipSuccess ? KVG_OK : KVG_E_HIP; }

}  // namespace host
}  // namespace kvg
