// C ABI of the packed sequences' calls (declarations and contracts in include/kvg.h).
#include "kvg_packed_host.h"

namespace {

using namespace kvg::host;
using kvg::fits_grid;

// The tiles' launch, the few kernel's, and the fold of those that are split.
int attn_launch(kvg::PackedAttnArgs a, const AttnPlan& plan, int32_t dtype, char* ws, hipStream_t stream) {
  a.few_rows = (int32_t)plan.few_rows;
  a.n_tiles = (int32_t)plan.n_tiles;
  kvg::PackedAttnArgs few = a, tiles = a;
  few.part = {reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + plan.few_ml), plan.few_seg};
  ws += plan.few_ml + plan.few_acc;
  tiles.part = {reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + plan.tile_ml), plan.tile_seg};
  int st = KVG_OK;
  if (a.n_tiles > 0)
    st = hip_status(dtype == KVG_F32 ? kvg::launch_packed_f32(tiles, stream) : kvg::launch_packed_tiles(tiles, dtype, stream));
  if (st == KVG_OK && a.few_rows > 0) st = hip_status(kvg::launch_packed_few(few, dtype, stream));
  if (st == KVG_OK && (plan.tile_seg > 1 || plan.few_seg > 1))
    st = hip_status(kvg::launch_packed_fold(tiles, few.part, dtype, stream));
  return st;
}

// kvg_rotate, and kvg_rotate_axes (axes given, positions NULL)
int rotate(const kvg_rotary* rotary, const kvg_axes* axes, int32_t dtype, int32_t head_dim, int32_t n_tokens, int32_t n_heads,
           const int64_t* positions, const void* x, int64_t x_stride, void* y, int64_t y_stride, void* stream) {
  if (dtype != KVG_F32 && dtype != KVG_BF16) return KVG_E_DTYPE;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return KVG_E_SHAPE;
  int st = check_rotary(rotary, head_dim);
  if (st != KVG_OK) return st;
  if (axes != nullptr && (st = check_axes(rotary, head_dim, axes, n_tokens)) != KVG_OK) return st;
  if (n_tokens < 0 || n_heads <= 0 || (int64_t)n_heads * head_dim > INT32_MAX) return KVG_E_INVAL;
  kvg::RotateArgs a;
  const int64_t dense = (int64_t)n_heads * head_dim;
  if ((st = check_stride(x_stride, dense, raw_bytes(dtype), &a.x_stride)) != KVG_OK) return st;
  if ((st = check_stride(y_stride, dense, raw_bytes(dtype), &a.y_stride)) != KVG_OK) return st;
  if (n_tokens == 0) return KVG_OK;
  if ((axes == nullptr && positions == nullptr) || x == nullptr || y == nullptr) return KVG_E_INVAL;
  if (x == y && a.x_stride != a.y_stride) return KVG_E_INVAL;
  if (!aligned16(x) || !aligned16(y)) return KVG_E_ALIGN;
  if (!fits_grid(n_tokens, 256)) return KVG_E_SHAPE;
  a.x = x;
  a.y = y;
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.n_heads = n_heads;
  a.D = head_dim;
  fill_rotary(rotary, head_dim, &a.rot);
  kvg::AxesArgs turn;
  if (axes != nullptr) fill_axes(rotary, axes, &a.rot, &turn);
  return hip_status(kvg::launch_rotate(a, axes != nullptr ? &turn : nullptr, dtype, static_cast<hipStream_t>(stream)));
}

// kvg_norm_append, and kvg_norm_append_axes (axes given)
int norm_append(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, const kvg_rotary* rotary,
                const kvg_axes* axes, const kvg_head_norm* norm, int32_t layer0, int32_t n_layers, const void* q_raw,
                const void* k_raw, const void* v_raw, void* q_out, void* stream) {
  int st = check_cache(cache);
  if (st != KVG_OK) return st;
  if ((st = check_rotary(rotary, cache->head_dim)) != KVG_OK) return st;
  if ((st = check_layers(cache, layer0, n_layers)) != KVG_OK) return st;
  if ((st = check_packed(cache, seqs, packed)) != KVG_OK) return st;
  if (axes != nullptr && (st = check_axes(rotary, cache->head_dim, axes, packed->n_tokens)) != KVG_OK) return st;
  if (norm != nullptr && (!(norm->eps >= 0.0f) || !std::isfinite(norm->eps) || !std::isfinite(norm->weight_offset)))
    return KVG_E_INVAL;
  kvg::NormAppendArgs a;
  std::memset(&a, 0, sizeof(a));
  const size_t raw = raw_bytes(cache->dtype);
  const int64_t q_dense = (int64_t)cache->n_q_heads * cache->head_dim, kv_dense = (int64_t)cache->n_kv_heads * cache->head_dim;
  if ((st = check_stride(packed->q_stride, q_dense, raw, &a.q_stride)) != KVG_OK) return st;
  if ((st = check_stride(packed->k_stride, kv_dense, raw, &a.k_stride)) != KVG_OK) return st;
  if ((st = check_stride(packed->v_stride, kv_dense, raw, &a.v_stride)) != KVG_OK) return st;
  if ((q_raw == nullptr) != (q_out == nullptr)) return KVG_E_INVAL;
  if (packed->n_tokens == 0 || packed->max_len == 0) return KVG_OK;
  if (k_raw == nullptr || v_raw == nullptr || (q_raw != nullptr && q_raw == q_out && a.q_stride != q_dense)) return KVG_E_INVAL;
  const void* w_q = norm != nullptr ? norm->q_weight : nullptr;
  const void* w_k = norm != nullptr ? norm->k_weight : nullptr;
  if (!aligned16(q_raw) || !aligned16(k_raw) || !aligned16(v_raw) || !aligned16(q_out) || !aligned16(w_q) || !aligned16(w_k) ||
      !aligned16(cache->k_pool) || !aligned16(cache->v_pool))
    return KVG_E_ALIGN;
  if (!fits_grid(packed->n_tokens, 256)) return KVG_E_SHAPE;
  a.seqs = packed_seqs(seqs, packed);
  a.start_pos = seqs->start_pos;
  a.k_pool = cache->k_pool;
  a.v_pool = cache->v_pool;
  a.layer_elems = layer_elems(cache);
  a.n_pages = cache->n_pages;
  a.q_raw = q_raw;
  a.k_raw = k_raw;
  a.v_raw = v_raw;
  a.q_out = q_out;
  a.q_weight = w_q;
  a.k_weight = w_k;
  a.eps = norm != nullptr ? norm->eps : 0.0f;
  a.weight_offset = norm != nullptr ? norm->weight_offset : 0.0f;
  a.Hq = cache->n_q_heads;
  a.Hkv = cache->n_kv_heads;
  a.D = cache->head_dim;
  a.layer0 = layer0;
  a.n_layers = n_layers;
  fill_rotary(rotary, cache->head_dim, &a.rot);
  kvg::AxesArgs turn;
  if (axes != nullptr) fill_axes(rotary, axes, &a.rot, &turn);
  return hip_status(kvg::launch_norm_append(a, axes != nullptr ? &turn : nullptr, cache->dtype, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int kvg_rotary_frequencies(const kvg_rotary* rotary, int32_t head_dim, double* theta_out) {
  if (theta_out == nullptr) return KVG_E_INVAL;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return KVG_E_SHAPE;
  const int st = check_rotary(rotary, head_dim);
  if (st == KVG_OK) frequencies(rotary, rotary_dim(rotary, head_dim), theta_out);
  return st;
}

int kvg_artifact_header_init_rotary(const kvg_cache* cache, int32_t n_tokens, int64_t own_pos, const kvg_rotary* rotary,
                                    kvg_artifact_hdr* hdr) {
  int st = check_cache(cache);
  if (st != KVG_OK) return st;
  if ((st = check_rotary(rotary, cache->head_dim)) != KVG_OK) return st;
  const int dim = rotary_dim(rotary, cache->head_dim);
  const double base = scaled_base(rotary, dim);
  const bool one_base = rotary->scaling == KVG_ROTARY_PLAIN || rotary->scaling == KVG_ROTARY_BASE || rotary->factor == 1.0;
  const kvg_rope rope = {std::isfinite(base) ? base : rotary->base, rotary->pairing, 0};
  st = kvg_artifact_header_init(cache, n_tokens, own_pos, &rope, hdr);
  if (st == KVG_OK && (!one_base || dim != cache->head_dim || !std::isfinite(base))) hdr->rope_pairing = KVG_ROPE_OTHER;
  return st;
}

int kvg_rotate(const kvg_rotary* rotary, int32_t dtype, int32_t head_dim, int32_t n_tokens, int32_t n_heads,
               const int64_t* positions, const void* x, int64_t x_stride, void* y, int64_t y_stride, void* stream) {
  return rotate(rotary, nullptr, dtype, head_dim, n_tokens, n_heads, positions, x, x_stride, y, y_stride, stream);
}

int kvg_rotate_axes(const kvg_rotary* rotary, const kvg_axes* axes, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                    int32_t n_heads, const void* x, int64_t x_stride, void* y, int64_t y_stride, void* stream) {
  if (axes == nullptr) return KVG_E_INVAL;
  return rotate(rotary, axes, dtype, head_dim, n_tokens, n_heads, nullptr, x, x_stride, y, y_stride, stream);
}

int kvg_norm_append(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, const kvg_rotary* rotary,
                    const kvg_head_norm* norm, int32_t layer0, int32_t n_layers, const void* q_raw, const void* k_raw,
                    const void* v_raw, void* q_out, void* stream) {
  return norm_append(cache, seqs, packed, rotary, nullptr, norm, layer0, n_layers, q_raw, k_raw, v_raw, q_out, stream);
}

int kvg_norm_append_axes(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, const kvg_rotary* rotary,
                         const kvg_axes* axes, const kvg_head_norm* norm, int32_t layer0, int32_t n_layers, const void* q_raw,
                         const void* k_raw, const void* v_raw, void* q_out, void* stream) {
  if (axes == nullptr) return KVG_E_INVAL;
  return norm_append(cache, seqs, packed, rotary, axes, norm, layer0, n_layers, q_raw, k_raw, v_raw, q_out, stream);
}

size_t kvg_packed_attn_workspace_bytes(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed,
                                       int32_t n_layers) {
  if (check_cache(cache) != KVG_OK || check_packed(cache, seqs, packed) != KVG_OK || n_layers <= 0 ||
      n_layers > cache->n_layers)
    return 0;
  // whichever layers the call is for
  size_t most = 0;
  const bool windowed = cache->layer_window != nullptr;
  for (int32_t l = 0; l <= (windowed ? cache->n_layers - n_layers : 0); ++l) {
    const AttnPlan plan = attn_plan(cache, seqs, packed, n_layers, windowed ? cache->layer_window + l : nullptr);
    if (!plan.fits) return 0;
    most = std::max(most, plan.total());
  }
  return most;
}

int kvg_packed_attn(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, int32_t layer0, int32_t n_layers,
                    const void* q, float scale, void* out, void* ws, size_t ws_bytes, void* stream) {
  int st = check_cache(cache);
  if (st != KVG_OK) return st;
  if ((st = check_layers(cache, layer0, n_layers)) != KVG_OK) return st;
  if ((st = check_packed(cache, seqs, packed)) != KVG_OK) return st;
  const float scale_log2 = scale * 1.4426950408889634f;
  if (!(scale > 0.0f) || !std::isfinite(scale_log2)) return KVG_E_INVAL;      // scores go in log2 units
  kvg::PackedAttnArgs a;
  std::memset(&a, 0, sizeof(a));
  if ((st = check_stride(packed->q_stride, (int64_t)cache->n_q_heads * cache->head_dim, raw_bytes(cache->dtype),
                         &a.q_stride)) != KVG_OK)
    return st;
  if ((st = fill_windows(cache, layer0, n_layers, a.window)) != KVG_OK) return st;
  // the caller's array, as the size query reads it: a launch carries kMaxWindowLayers windows, a call without any may
  // have more layers
  const AttnPlan plan = attn_plan(cache, seqs, packed, n_layers, cache->layer_window != nullptr ? cache->layer_window + layer0 : nullptr);
  if (!plan.fits || !fits_grid(packed->n_tokens, 256)) return KVG_E_SHAPE;
  if (ws == nullptr || ws_bytes < plan.total()) return KVG_E_WORKSPACE;
  if (packed->n_tokens == 0 || packed->max_len == 0) return KVG_OK;
  if (q == nullptr || out == nullptr || q == out) return KVG_E_INVAL;
  if (!aligned16(q) || !aligned16(out) || !aligned16(ws) || !aligned16(cache->k_pool) || !aligned16(cache->v_pool))
    return KVG_E_ALIGN;
  a.seqs = packed_seqs(seqs, packed);
  a.k_pool = cache->k_pool;
  a.v_pool = cache->v_pool;
  a.layer_elems = layer_elems(cache);
  a.n_pages = cache->n_pages;
  a.q = q;
  a.out = out;
  a.scale_log2 = scale_log2;
  a.Hq = cache->n_q_heads;
  a.Hkv = cache->n_kv_heads;
  a.D = cache->head_dim;
  a.group = cache->n_q_heads / cache->n_kv_heads;
  a.layer0 = layer0;
  a.n_layers = n_layers;
  return attn_launch(a, plan, cache->dtype, static_cast<char*>(ws), static_cast<hipStream_t>(stream));
}

}  // extern "C"
