// C ABI of the packed sequences' calls (declarations and contracts in include/kvg.h).
#include "kvg_packed_host.h"

namespace {

using namespace kvg::host;
using kvg::fits_grid;

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
  kvg::NormAppendArgs a;
  kvg::AxesArgs turn;
  bool empty = false;
  st = append_args(cache, seqs, packed, rotary, axes, norm, layer0, n_layers, q_raw, k_raw, v_raw, q_out, &a, &turn, &empty);
  if (st != KVG_OK || empty) return st;
  if (!fits_grid(packed->n_tokens, 256)) return KVG_E_SHAPE;
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

int kvg_artifact_header_init_axes(const kvg_cache* cache, int32_t n_tokens, int64_t own_pos, const kvg_rotary* rotary,
                                  const kvg_axes* axes, kvg_artifact_hdr* hdr) {
  int st = check_cache(cache);
  if (st != KVG_OK) return st;
  if ((st = check_rotary(rotary, cache->head_dim)) != KVG_OK) return st;
  if ((st = check_axes(rotary, cache->head_dim, axes, 0)) != KVG_OK) return st;
  const kvg_rope rope = {rotary->base, rotary->pairing, 0};
  st = kvg_artifact_header_init(cache, n_tokens, own_pos, &rope, hdr);
  if (st == KVG_OK) hdr->rope_pairing = KVG_ROPE_OTHER;
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
  return check_cache(cache) == KVG_OK ? attn_workspace_bytes(cache, seqs, packed, n_layers) : 0;
}

int kvg_packed_attn(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, int32_t layer0, int32_t n_layers,
                    const void* q, float scale, void* out, void* ws, size_t ws_bytes, void* stream) {
  int st = check_cache(cache);
  if (st != KVG_OK) return st;
  kvg::PackedAttnArgs a;
  AttnPlan plan;
  bool empty = false;
  st = attn_args(cache, seqs, packed, layer0, n_layers, q, scale, out, ws, ws_bytes, &a, &plan, &empty);
  if (st != KVG_OK || empty) return st;
  const int32_t dtype = cache->dtype;
  return attn_launch(
      a, plan, dtype, static_cast<char*>(ws), static_cast<hipStream_t>(stream),
      [dtype](const kvg::PackedAttnArgs& t, hipStream_t s) {
        return dtype == KVG_F32 ? kvg::launch_packed_f32(t, s) : kvg::launch_packed_tiles(t, dtype, s);
      },
      [dtype](const kvg::PackedAttnArgs& t, hipStream_t s) { return kvg::launch_packed_few(t, dtype, s); });
}

}  // extern "C"
