// C ABI of the 8-bit integer caches (declarations and contracts in include/kvg.h).
#include "kvg_int8.h"
#include "kvg_packed_host.h"

namespace {

using namespace kvg::host;
using kvg::fits_grid;

size_t block_pages(const kvg_int8_cache* c, int32_t n_tokens) {
  return ((size_t)n_tokens + c->pages.page_size - 1) / c->pages.page_size;
}

// bytes of a block's integers, which its scales follow
size_t block_integers(const kvg_int8_cache* c, int32_t n_tokens) {
  return (size_t)c->pages.n_layers * 2 * block_pages(c, n_tokens) * c->pages.n_kv_heads * c->pages.page_size * c->pages.head_dim;
}

// The copies of a block's integers and of its scales, between the pages and `payload`; a deposit or a graft.
int block_copy(const kvg_int8_cache* cache, const int32_t* block_table, int32_t table_len, int32_t first_token, int32_t n_tokens,
               void* payload, bool deposit, hipStream_t stream) {
  const kvg_cache& c = cache->pages;
  if (first_token % c.page_size != 0) return KVG_E_ALIGN;
  const int64_t n_pages = (int64_t)block_pages(cache, n_tokens);
  if ((int64_t)first_token / c.page_size + n_pages > table_len) return KVG_E_CAPACITY;
  if (!aligned16(payload) || !aligned16(c.k_pool) || !aligned16(c.v_pool)) return KVG_E_ALIGN;
  kvg::CopyArgs a;
  std::memset(&a, 0, sizeof(a));
  a.k_pool = c.k_pool;
  a.v_pool = c.v_pool;
  a.page_bytes = (int64_t)c.n_kv_heads * c.page_size * c.head_dim;
  a.layer_bytes = c.n_pages * a.page_bytes;
  a.n_pages = c.n_pages;
  a.block_table = block_table;
  a.payload = payload;
  a.first_page = first_token / c.page_size;
  a.n_block_pages = (int32_t)n_pages;
  a.n_tokens = n_tokens;
  a.n_layers = c.n_layers;
  a.row_bytes = c.head_dim;
  a.Hkv = c.n_kv_heads;
  a.D = c.head_dim;
  const kvg::Int8ScaleCopyArgs s = {{cache->k_scale, cache->v_scale}, c.n_pages, block_table,
                                    reinterpret_cast<float*>(static_cast<char*>(payload) + block_integers(cache, n_tokens)),
                                    a.first_page, a.n_block_pages, c.n_layers, c.n_kv_heads};
  // the byte moves of an fp8 cache of this geometry
  if (!fits_grid(kvg::copy_workgroups(a, KVG_FP8_E4M3), 256) || !fits_grid((kvg::int8_scale_values(s) + 255) / 256, 256)) return KVG_E_SHAPE;
  int st = hip_status(deposit ? kvg::launch_deposit(a, stream) : kvg::launch_graft(a, KVG_FP8_E4M3, stream));
  if (st == KVG_OK) st = hip_status(kvg::launch_int8_scales(s, deposit, stream));
  return st;
}

}  // namespace

extern "C" {

int kvg_int8_append(const kvg_int8_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, const kvg_rotary* rotary,
                    const kvg_axes* axes, const kvg_head_norm* norm, int32_t layer0, int32_t n_layers, const void* q_raw,
                    const void* k_raw, const void* v_raw, void* q_out, void* stream) {
  int st = check_int8_cache(cache);
  if (st != KVG_OK) return st;
  kvg::NormAppendArgs a;
  kvg::AxesArgs turn;
  bool empty = false;
  st = append_args(&cache->pages, seqs, packed, rotary, axes, norm, layer0, n_layers, q_raw, k_raw, v_raw, q_out, &a, &turn, &empty);
  if (st != KVG_OK || empty) return st;
  if (!fits_grid(kvg::int8_append_units(a.seqs), 256)) return KVG_E_SHAPE;
  return hip_status(kvg::launch_int8_append(a, {cache->k_scale, cache->v_scale}, axes != nullptr ? &turn : nullptr,
                                            static_cast<hipStream_t>(stream)));
}

size_t kvg_int8_attn_workspace_bytes(const kvg_int8_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed,
                                     int32_t n_layers) {
  return check_int8_cache(cache) == KVG_OK ? attn_workspace_bytes(&cache->pages, seqs, packed, n_layers) : 0;
}

int kvg_int8_attn(const kvg_int8_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, int32_t layer0,
                  int32_t n_layers, const void* q, float scale, void* out, void* ws, size_t ws_bytes, void* stream) {
  int st = check_int8_cache(cache);
  if (st != KVG_OK) return st;
  kvg::PackedAttnArgs a;
  AttnPlan plan;
  bool empty = false;
  st = attn_args(&cache->pages, seqs, packed, layer0, n_layers, q, scale, out, ws, ws_bytes, &a, &plan, &empty);
  if (st != KVG_OK || empty) return st;
  const kvg::Int8Scales scales = {cache->k_scale, cache->v_scale};
  return attn_launch(
      a, plan, KVG_BF16, static_cast<char*>(ws), static_cast<hipStream_t>(stream),
      [&](const kvg::PackedAttnArgs& t, hipStream_t s) { return kvg::launch_int8_tiles(t, scales, s); },
      [&](const kvg::PackedAttnArgs& t, hipStream_t s) { return kvg::launch_int8_few(t, scales, s); });
}

size_t kvg_int8_payload_bytes(const kvg_int8_cache* cache, int32_t n_tokens) {
  if (check_int8_cache(cache) != KVG_OK || n_tokens <= 0) return 0;
  return block_integers(cache, n_tokens) +
         (size_t)cache->pages.n_layers * 2 * block_pages(cache, n_tokens) * cache->pages.n_kv_heads * sizeof(float);
}

int kvg_int8_header_init(const kvg_int8_cache* cache, int32_t n_tokens, int64_t own_pos, kvg_artifact_hdr* hdr) {
  const int st = check_int8_cache(cache);
  if (st != KVG_OK) return st;
  if (hdr == nullptr || n_tokens <= 0) return KVG_E_INVAL;
  std::memset(hdr, 0, sizeof(*hdr));
  hdr->magic = KVG_ARTIFACT_MAGIC;
  hdr->version = KVG_ARTIFACT_VERSION;
  hdr->dtype = KVG_INT8;
  hdr->n_layers = cache->pages.n_layers;
  hdr->n_kv_heads = cache->pages.n_kv_heads;
  hdr->head_dim = cache->pages.head_dim;
  hdr->page_size = cache->pages.page_size;
  hdr->n_tokens = n_tokens;
  hdr->own_pos = own_pos;
  hdr->rope_base = 1.0;
  hdr->rope_pairing = KVG_ROPE_OTHER;
  hdr->payload_bytes = kvg_int8_payload_bytes(cache, n_tokens);
  return KVG_OK;
}

int kvg_int8_deposit(const kvg_int8_cache* cache, const int32_t* block_table, int32_t table_len, int32_t first_token,
                     int32_t n_tokens, void* payload, void* stream) {
  const int st = check_int8_cache(cache);
  if (st != KVG_OK) return st;
  if (block_table == nullptr || payload == nullptr || n_tokens <= 0 || first_token < 0 || table_len <= 0) return KVG_E_INVAL;
  return block_copy(cache, block_table, table_len, first_token, n_tokens, payload, true, static_cast<hipStream_t>(stream));
}

int kvg_int8_graft(const kvg_int8_cache* cache, const kvg_artifact_hdr* hdr, const void* payload, const int32_t* block_table,
                   int32_t table_len, int32_t first_token, int64_t target_pos, void* stream) {
  const int st = check_int8_cache(cache);
  if (st != KVG_OK) return st;
  if (hdr == nullptr || payload == nullptr || block_table == nullptr || first_token < 0 || table_len <= 0) return KVG_E_INVAL;
  if (hdr->magic != KVG_ARTIFACT_MAGIC || hdr->version != KVG_ARTIFACT_VERSION || hdr->n_tokens <= 0) return KVG_E_CORRUPT;
  if (hdr->dtype != KVG_INT8) return KVG_E_DTYPE;
  const kvg_cache& c = cache->pages;
  if (hdr->n_layers != c.n_layers || hdr->n_kv_heads != c.n_kv_heads || hdr->head_dim != c.head_dim || hdr->page_size != c.page_size)
    return KVG_E_SHAPE;
  if (hdr->payload_bytes != kvg_int8_payload_bytes(cache, hdr->n_tokens) || hdr->rope_pairing != KVG_ROPE_OTHER) return KVG_E_CORRUPT;
  if (target_pos != hdr->own_pos) return KVG_E_POSITION;
  return block_copy(cache, block_table, table_len, first_token, hdr->n_tokens, const_cast<void*>(payload), false,
                    static_cast<hipStream_t>(stream));
}

}  // extern "C"
