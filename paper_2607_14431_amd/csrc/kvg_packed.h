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

// A sequence, its range, and the place of a searched unit in it: unit `at` of its `count`; b -1: no sequence.
struct SeqUnit {
  int b, at, count;
  SeqRange range;
};

// Unit `target` of the batch, whose sequences have count(range) units each.  All lanes of a wave search together, 64
// sequences at a time, each lane reading one; the result is uniform.
template <typename Count>
__device__ __forceinline__ SeqUnit find_unit(const PackedSeqs& s, int target, Count count) {
  const int lane = __lane_id();
  for (int b0 = 0; b0 < s.batch; b0 += 64) {
    const int b = b0 + lane;
    const SeqRange r = b < s.batch ? seq_range(s, b) : SeqRange{0, 0, 0};
    const int n = count(r);
    int sum = n;                                           // of this lane's sequence and those before it
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int before = __shfl_up(sum, d);
      sum += lane >= d ? before : 0;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(sum > target);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      const int c = __builtin_amdgcn_readlane(n, at);
      return {b0 + at, target - (__builtin_amdgcn_readlane(sum, at) - c), c,
              {__builtin_amdgcn_readlane(r.row0, at), __builtin_amdgcn_readlane(r.len, at), __builtin_amdgcn_readlane(r.ctx, at)}};
    }
    target -= __builtin_amdgcn_readlane(sum, 63);
  }
  return {-1, 0, 0, {0, 0, 0}};
}

// The sequence of packed row `tok` and its place there.
__device__ __forceinline__ SeqUnit find_token(const PackedSeqs& s, int tok) {
  const int lane = __lane_id();
  for (int b0 = 0; b0 < s.batch; b0 += 64) {
    const int b = b0 + lane;
    const SeqRange r = b < s.batch ? seq_range(s, b) : SeqRange{0, 0, 0};
    const uint64_t mine = __builtin_amdgcn_ballot_w64(tok >= r.row0 && tok - r.row0 < r.len);
    if (mine != 0) {
      const int at = __builtin_ctzll(mine);
      const int row0 = __builtin_amdgcn_readlane(r.row0, at), len = __builtin_amdgcn_readlane(r.len, at);
      return {b0 + at, tok - row0, len, {row0, len, __builtin_amdgcn_readlane(r.ctx, at)}};
    }
  }
  return {-1, 0, 0, {0, 0, 0}};
}

// Keys of a segment of the attention's sums (absolute multiples of the logical index).  Short ones spread few rows over the
// chip, long ones fold less.  256 / 512 / 1,024 keys, us: one token over 4.6k keys 20 / 24 / 35, 16 over 33k 579 / 531 / 523,
// chunks of 35 rows over 32k (fp8) 181 / 145 / 124, a mixed batch with a window of 1,024 175 / 164 / 196, ragged fp32 chunks over
// 1k 37 / 33 / 54, eight prompts 478 / 475 / 465, 12,288 tokens 1,211 / 1,159 / 1,132.
constexpr int kPackedSeg = 512;

// The rotation of a launch: frequencies and what cos and sin are multiplied with.
struct RotaryArgs {
  int32_t pairing, dim;       // dim: components rotated
  double amplitude;
  double theta[kMaxHalfDim];
};

// Positions with several axes: the axis of each pair, and [axes][rows] positions.
struct AxesArgs {
  const int64_t* positions;
  uint8_t axis[kMaxHalfDim];
};
struct NoAxes {};

struct RotateArgs {
  const void* x;
  void* y;
  int64_t x_stride, y_stride;
  const int64_t* positions;
  int32_t n_tokens, n_heads, D;
  int32_t steps;              // of a workgroup (set by the launcher)
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
  int32_t Hq, Hkv, D, layer0, n_layers;
  int32_t layers_per_block, steps;      // of a workgroup (set by the launcher)
  RotaryArgs rot;
};

// Partials of a launch over n_seg segments: a (reference, sum) and D sums per pair and segment.
struct PackedPartials {
  float* ml;
  float* acc;
  int32_t n_seg;              // 1: the launch is not split
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
  // Sequences go in tiles of (row, query head) pairs of a KV head (n_tiles: a bound of the batch's); in bf16 and fp8 caches
  // those of at most kFewPairs pairs are the few kernel's where it runs (few_rows > 0: a bound of their rows).
  // Where a split launch leaves its partials: the few kernel [n_layers][rows][Hq][n_seg], rows counted over its own
  // sequences; tiles in blocks of 32 pairs (part_block).
  int32_t few_rows, n_tiles;
  PackedPartials part;
  int32_t window[kMaxWindowLayers];
};

// axes: null where a token has one position
hipError_t launch_rotate(const RotateArgs& a, const AxesArgs* axes, int dtype, hipStream_t stream);
hipError_t launch_norm_append(const NormAppendArgs& a, const AxesArgs* axes, int dtype, hipStream_t stream);
// bf16 and fp8 caches: pairs of a tile, workgroups of the launches
constexpr int kFewPairs = 32;
__device__ __forceinline__ bool is_few(const PackedAttnArgs& a, const SeqRange& s) {
  return a.few_rows > 0 && (int64_t)s.len * a.group <= kFewPairs;
}
constexpr int kTilePairs = 128;
inline int64_t packed_tile_workgroups(const PackedAttnArgs& a) { return (int64_t)a.n_layers * a.part.n_seg * a.n_tiles * a.Hkv; }
inline int64_t packed_few_workgroups(const PackedAttnArgs& a) { return (int64_t)a.n_layers * a.part.n_seg * a.seqs.batch * a.Hkv; }
hipError_t launch_packed_tiles(const PackedAttnArgs& a, int dtype, hipStream_t stream);
hipError_t launch_packed_few(const PackedAttnArgs& a, int dtype, hipStream_t stream);
// out = the segments of the split launches, folded in order: of the tiles (a.part) and of the few kernel
inline int64_t packed_fold_workgroups(const PackedAttnArgs& a, int pairs) {
  return (int64_t)a.n_layers * a.n_tiles * a.Hkv * (pairs / 32) * (a.D / 32);
}
hipError_t launch_packed_fold(const PackedAttnArgs& a, const PackedPartials& few, int dtype, hipStream_t stream);
// fp32 caches: tiles of kF32Pairs pairs
constexpr int kF32Pairs = 32;
hipError_t launch_packed_f32(const PackedAttnArgs& a, hipStream_t stream);

}  // namespace kvg
