// Packed sequences: kernel parameter blocks, launchers, and the search of a packed row's sequence.
#pragma once

#include <hip/hip_runtime.h>

#include "kvg_device.h"

namespace kvg {

// A batch of packed sequences over a paged cache (kvg_seqs and kvg_packed).
struct PackedSeqs {
  const int32_t* cu;          // [batch + 1]
  const int32_t* ctx_lens;    // [batch]
  const int32_t* tables;      // [batch][max_pages]
  int32_t batch, n_tokens, max_len, max_ctx_len, max_pages;
};

// Sequence b's new tokens: rows [row0, row0 + len) at logical indices ctx + 0, 1, ...; len 0 for a sequence
// that has none or whose metadata is not as kvg_packed demands.
struct SeqRange {
  int row0, len, ctx;
};
__device__ __forceinline__ SeqRange seq_range(const PackedSeqs& s, int b) {
  const int r0 = s.cu[b], r1 = s.cu[b + 1], ctx = s.ctx_lens[b];
  const int64_t len = (int64_t)r1 - r0;
  const bool ok = r0 >= 0 && r1 <= s.n_tokens && len >= 0 && len <= s.max_len && ctx >= 0 && ctx <= s.max_ctx_len &&
                  ctx + len <= (int64_t)s.max_pages * kPage;
  return {r0, ok ? (int)len : 0, ctx};
}

// The rotation of a launch: frequencies and what cos and sin are multiplied with.
struct RotaryArgs {
  int32_t pairing, dim;       // dim: components rotated
  double amplitude;
  double theta[kMaxHalfDim];
};

struct RotateArgs {
  const void* x;
  void* y;
  int64_t x_stride, y_stride;
  const int64_t* positions;
  int32_t n_tokens, n_heads, D;
  RotaryArgs rot;
};

struct NormAppendArgs {
  PackedSeqs seqs;
  const int64_t* start_pos;
  void* k_pool;
  void* v_pool;
  int64_t layer_elems, n_pages;
  const void* q_raw;          // or null
  const void* k_raw;
  const void* v_raw;
  void* q_out;
  int64_t q_stride, k_stride, v_stride;
  const void* q_weight;       // or null: no norm
  const void* k_weight;
  float eps, weight_offset;
  int32_t Hq, Hkv, D, layer0, n_layers, layers_per_block;
  RotaryArgs rot;
};

struct PackedAttnArgs {
  PackedSeqs seqs;
  const void* k_pool;
  const void* v_pool;
  int64_t layer_elems, n_pages;
  const void* q;              // [n_layers][n_tokens][q_stride] raw dtype
  void* out;                  // [n_layers][n_tokens][Hq][D] raw dtype
  int64_t q_stride;
  float scale_log2;
  int32_t Hq, Hkv, D, group, layer0, n_layers;
  int32_t window[kMaxWindowLayers];
};

hipError_t launch_rotate(const RotateArgs& a, int dtype, hipStream_t stream);
hipError_t launch_norm_append(const NormAppendArgs& a, int dtype, hipStream_t stream);
hipError_t launch_packed_attn(const PackedAttnArgs& a, int dtype, hipStream_t stream);

}  // namespace kvg
