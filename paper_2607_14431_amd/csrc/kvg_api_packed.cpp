// C ABI of the packed sequences' calls (declarations and contracts in include/kvg.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "kvg.h"
#include "kvg_host.h"
#include "kvg_launch.h"
#include "kvg_packed.h"

namespace {

using namespace kvg::host;
using kvg::fits_grid;

constexpr double kTwoPi = 6.283185307179586476925;

int rotary_dim(const kvg_rotary* r, int32_t head_dim) { return r->rotary_dim == 0 ? head_dim : r->rotary_dim; }

bool positive(double x) { return x > 0.0 && std::isfinite(x); }

int check_rotary(const kvg_rotary* r, int32_t head_dim) {
  if (r == nullptr || !(r->base > 1.0) || !std::isfinite(r->base) || !positive(r->amplitude) || r->reserved != 0)
    return KVG_E_INVAL;
  if (r->pairing != KVG_ROPE_HALF && r->pairing != KVG_ROPE_INTERLEAVED) return KVG_E_INVAL;
  if (r->scaling < KVG_ROTARY_PLAIN || r->scaling > KVG_ROTARY_INDEX) return KVG_E_INVAL;
  if (r->scaling != KVG_ROTARY_PLAIN && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) return KVG_E_INVAL;
  if ((r->scaling == KVG_ROTARY_ROTATIONS || r->scaling == KVG_ROTARY_INDEX) &&
      (!positive(r->original_len) || !positive(r->fast) || !positive(r->slow) || !(r->fast > r->slow)))
    return KVG_E_INVAL;
  if (r->rotary_dim < 0 || r->rotary_dim > head_dim || r->rotary_dim % 16 != 0) return KVG_E_SHAPE;
  return KVG_OK;
}

double scaled_base(const kvg_rotary* r, int dim) {
  return r->scaling == KVG_ROTARY_BASE ? r->base * std::pow(r->factor, dim / (dim - 2.0)) : r->base;
}

void frequencies(const kvg_rotary* r, int dim, double* theta) {
  const double base = scaled_base(r, dim);
  double lo = 0.0, hi = 0.0;
  if (r->scaling == KVG_ROTARY_INDEX) {
    auto index = [&](double turns) { return dim * std::log(r->original_len / (kTwoPi * turns)) / (2.0 * std::log(r->base)); };
    lo = std::max(std::floor(index(r->fast)), 0.0);
    hi = std::min(std::ceil(index(r->slow)), dim - 1.0);
  }
  for (int i = 0; i < dim / 2; ++i) {
    const double t = std::pow(base, -2.0 * i / dim);
    double keep = 1.0;                                   // share of the unscaled frequency
    if (r->scaling == KVG_ROTARY_LINEAR)
      keep = 0.0;
    else if (r->scaling == KVG_ROTARY_ROTATIONS)
      keep = std::clamp((r->original_len * t / kTwoPi - r->slow) / (r->fast - r->slow), 0.0, 1.0);
    else if (r->scaling == KVG_ROTARY_INDEX)
      keep = 1.0 - std::clamp((i - lo) / std::max(hi - lo, 0.001), 0.0, 1.0);
    theta[i] = keep == 1.0 ? t : t * keep + t / r->factor * (1.0 - keep);
  }
}

// The rotary as a launch carries it.  Each thread keeps its last one: a model has one or two, and its powers
// are a good part of a small call's time.
void fill_rotary(const kvg_rotary* r, int32_t head_dim, kvg::RotaryArgs* out) {
  thread_local kvg_rotary last = {};
  thread_local int last_dim = 0;
  thread_local kvg::RotaryArgs args;
  const int dim = rotary_dim(r, head_dim);
  if (dim != last_dim || std::memcmp(r, &last, sizeof(last)) != 0) {
    args.pairing = r->pairing;
    args.dim = dim;
    args.amplitude = r->amplitude;
    frequencies(r, dim, args.theta);
    last = *r;
    last_dim = dim;
  }
  out->pairing = args.pairing;
  out->dim = dim;
  out->amplitude = args.amplitude;
  std::memcpy(out->theta, args.theta, sizeof(double) * (dim / 2));
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

size_t raw_bytes(int32_t dtype) { return dtype == KVG_F32 ? 4 : 2; }

// A token stride in elements: `dense` for 0; KVG_E_INVAL when rows overlap, KVG_E_ALIGN when they leave 16 bytes.
int check_stride(int64_t stride, int64_t dense, size_t elem, int64_t* out) {
  *out = stride == 0 ? dense : stride;
  if (*out < dense) return KVG_E_INVAL;
  return *out * (int64_t)elem % 16 == 0 ? KVG_OK : KVG_E_ALIGN;
}

int check_packed(const kvg_cache* c, const kvg_seqs* s, const kvg_packed* p) {
  if (s == nullptr || s->block_tables == nullptr || s->ctx_lens == nullptr || s->start_pos == nullptr) return KVG_E_INVAL;
  if (p == nullptr || p->cu_tokens == nullptr || p->n_tokens < 0 || p->max_len < 0) return KVG_E_INVAL;
  if (s->batch <= 0 || s->max_pages <= 0 || s->max_ctx_len < 0) return KVG_E_INVAL;
  const int64_t room = (int64_t)s->max_pages * c->page_size;
  if (room > INT32_MAX - 2 * kvg::kPackedSeg) return KVG_E_SHAPE;      // a segment's end is an int
  if (s->max_ctx_len > room || p->max_len > room) return KVG_E_CAPACITY;
  return KVG_OK;
}

kvg::PackedSeqs packed_seqs(const kvg_seqs* s, const kvg_packed* p) {
  return {p->cu_tokens, s->ctx_lens, s->block_tables, s->batch, p->n_tokens, p->max_len, s->max_ctx_len, s->max_pages};
}

// A tile launch is split over segments when its workgroups (in units of the longest walk, `segs` segments) are few
// beside the chip and beside the segments: splitting shortens the walk, but every (row, segment) leaves D sums that are
// written and read again, more cheaply while the last-level cache holds them.  Measured, unsplit against split with its
// fold, us, at workgroups x segments.  bf16 and fp8, head_dim 256: 16 x 3 52 / 31, 40 x 9 116 / 53, 56 x 65 (fp8) 1,370
// / 493, 40 x 65 832 / 411, 64 x 33 445 / 302, 96 x 34 447 / 453, 104 x 3 46 / 53, 128 x 10 144 / 136, 128 x 34 456 /
// 571; 128: 64 x 33 334 / 134, 128 x 9 99 / 78, 128 x 33 357 / 294, 160 x 2 33 / 41, 184 x 12 128-134 / 96-122 (with
// and without windows), 192 x 4 35 / 51, 192 x 9 109 / 110, 192 x 34 363 / 442, 242 x 12 166 / 143, 250 x 4 51 / 60,
// 314 x 5 65 / 67, 388 x 12 167 / 189; 64: 54 x 35 271 / 63, 56 x 3 27 / 17, 88 x 13 98 / 49, 176 x 13 103 / 67, 250 x
// 40 330 / 280, 468 x 8 78 / 70.  fp32, more work on fewer rows to a workgroup: 32 x 2 26 / 21, 104 x 3 35 / 32, 184 x
// 3 45 / 34, 216 x 2 31 / 34, 256 x 5 73 / 81, 528 x 3 191 / 195.  The rule takes the slower side of two of
// these: 128 x 10 at 256 and 468 x 8 at 64.
bool split_tiles(bool f32, int64_t head_dim, int64_t workgroups, int64_t segs) {
  if (f32) return workgroups < std::min<int64_t>(256, 96 * (segs - 1));
  const bool cached = workgroups * segs * head_dim < 576000;           // partials of about 290 MB
  return workgroups < std::min<int64_t>({256, 48 * (segs - 1), (cached ? 32768 : 22528) / head_dim});
}

// Whether a split tile launch takes the short sequences too, whose own launch would have `workgroups`: one launch less, and its
// two stages of keys and values hide more of a small launch's waiting; large ones want the few kernel's smaller
// workgroups and no empty waves.  Few kernel against tiles, each with its fold, us, at workgroups.  bf16, head_dim 256: 80
// 26 / 24, 256 33 / 30, 512 52 / 56, 1,024 92 / 132, 8,448 536 / 1,090; 128: 128 23 / 21, 256 24 / 22, 512 31 / 32, 1,024 49 / 59; 64:
// 64 20 / 17, 256 24 / 17, 512 27 / 23.  fp8, 256: 64 21 / 24, 128 23 / 25, 256 26 / 27, 512 35 / 49; 128: 64 17 / 18, 256 29 / 23;
// 64: 16 19 / 16, 32 18 / 15.  One limit for all: at 512 it takes the slower side at head_dim 64.
bool few_in_tiles(const kvg_cache* c, int64_t workgroups) {
  return workgroups <= 256 && (c->dtype == KVG_BF16 || c->head_dim <= 128);
}

// How an attention call runs: rows of the few kernel and tiles at most, each launch's segments (1: not
// split), and where their partials lie in the workspace.
struct AttnPlan {
  int64_t few_rows, n_tiles;
  int32_t few_seg, tile_seg;
  size_t few_ml, few_acc, tile_ml, tile_acc;
  bool fits;                  // the launches, into a grid
  size_t total() const { return std::max(few_ml + few_acc + tile_ml + tile_acc, kAlign); }
};

// window: the n_layers layers' windows, or null.
AttnPlan attn_plan(const kvg_cache* c, const kvg_seqs* s, const kvg_packed* p, int32_t n_layers, const int32_t* window) {
  AttnPlan r = {0, 0, 1, 1, 0, 0, 0, 0, true};
  if (p->n_tokens == 0 || p->max_len == 0) return r;
  const bool f32 = c->dtype == KVG_F32;
  const int64_t group = c->n_q_heads / c->n_kv_heads, bm = f32 ? kvg::kF32Pairs : kvg::kTilePairs;
  const int64_t len = std::min(p->max_len, p->n_tokens);
  const int64_t keys = std::min((int64_t)s->max_ctx_len + p->max_len, (int64_t)s->max_pages * c->page_size);
  const int32_t segs = (int32_t)((keys + kvg::kPackedSeg - 1) / kvg::kPackedSeg);
  // all sequences in tiles; each sequence's round up
  const int64_t per_seq = (len * group + bm - 1) / bm;
  r.n_tiles = std::min(s->batch * per_seq, (p->n_tokens * group + (int64_t)std::min(s->batch, p->n_tokens) * (bm - 1)) / bm);
  int64_t longest = 0, sum = 0;                                        // segments of a layer's tile, about
  for (int l = 0; l < n_layers; ++l) {
    const int64_t W = window != nullptr ? window[l] : 0;
    const int64_t walk = W > 0 ? std::min<int64_t>(segs, (W + bm / group) / kvg::kPackedSeg + 1) : segs;
    longest = std::max(longest, walk);
    sum += walk;
  }
  if (split_tiles(f32, c->head_dim, r.n_tiles * c->n_kv_heads * sum / longest, longest)) r.tile_seg = segs;
  // The lengths are the device's.  A single sequence that may be long goes in tiles whatever its length.
  if (!f32 && (len * group <= kvg::kFewPairs || s->batch > 1) &&
      !(r.tile_seg > 1 && few_in_tiles(c, (int64_t)n_layers * segs * s->batch * c->n_kv_heads))) {
    r.few_rows = std::min<int64_t>(p->n_tokens, s->batch * std::min<int64_t>(len, kvg::kFewPairs / group));
    r.few_seg = segs;
    if (len * group <= kvg::kFewPairs) {
      r.n_tiles = 0;
      r.tile_seg = 1;
    }
  }
  const int64_t tile_grid = n_layers * r.n_tiles * c->n_kv_heads, fold_grid = (bm / 32) * (c->head_dim / 32);
  r.fits = fits_grid((int64_t)n_layers * r.few_seg * (r.few_rows > 0 ? s->batch : 0) * c->n_kv_heads, 256) &&
           fits_grid(tile_grid * r.tile_seg, 256) &&
           fits_grid(n_layers * r.few_rows * c->n_q_heads + (r.tile_seg > 1 ? tile_grid * fold_grid : 0), 256);
  if (!r.fits) return r;
  auto bytes = [&](int64_t row_heads, int32_t n_seg, size_t values) {
    return n_seg > 1 ? align_up((size_t)n_layers * row_heads * n_seg * values * sizeof(float)) : 0;
  };
  const int64_t few = r.few_rows * c->n_q_heads, tiles = r.n_tiles * c->n_kv_heads * bm;
  r.few_ml = bytes(few, r.few_seg, 2);
  r.few_acc = bytes(few, r.few_seg, c->head_dim);
  r.tile_ml = bytes(tiles, r.tile_seg, 2);
  r.tile_acc = bytes(tiles, r.tile_seg, c->head_dim);
  return r;
}

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
  if (dtype != KVG_F32 && dtype != KVG_BF16) return KVG_E_DTYPE;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return KVG_E_SHAPE;
  int st = check_rotary(rotary, head_dim);
  if (st != KVG_OK) return st;
  if (n_tokens < 0 || n_heads <= 0 || (int64_t)n_heads * head_dim > INT32_MAX) return KVG_E_INVAL;
  kvg::RotateArgs a;
  const int64_t dense = (int64_t)n_heads * head_dim;
  if ((st = check_stride(x_stride, dense, raw_bytes(dtype), &a.x_stride)) != KVG_OK) return st;
  if ((st = check_stride(y_stride, dense, raw_bytes(dtype), &a.y_stride)) != KVG_OK) return st;
  if (n_tokens == 0) return KVG_OK;
  if (positions == nullptr || x == nullptr || y == nullptr) return KVG_E_INVAL;
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
  return hip_status(kvg::launch_rotate(a, dtype, static_cast<hipStream_t>(stream)));
}

int kvg_norm_append(const kvg_cache* cache, const kvg_seqs* seqs, const kvg_packed* packed, const kvg_rotary* rotary,
                    const kvg_head_norm* norm, int32_t layer0, int32_t n_layers, const void* q_raw, const void* k_raw,
                    const void* v_raw, void* q_out, void* stream) {
  int st = check_cache(cache);
  if (st != KVG_OK) return st;
  if ((st = check_rotary(rotary, cache->head_dim)) != KVG_OK) return st;
  if ((st = check_layers(cache, layer0, n_layers)) != KVG_OK) return st;
  if ((st = check_packed(cache, seqs, packed)) != KVG_OK) return st;
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
  return hip_status(kvg::launch_norm_append(a, cache->dtype, static_cast<hipStream_t>(stream)));
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
