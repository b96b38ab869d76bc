// 8-bit integer caches with a scale for each page and KV head: kernel parameter blocks and launchers.
#pragma once

#include "kvg_packed.h"

namespace kvg {

// [n_layers][n_pages][Hkv] of the cache
struct Int8Scales {
  float* k;
  float* v;
};

// Stored integers are in [-kInt8Max, kInt8Max]; scales are 0 or at least kInt8Least, whose inverse is finite.
constexpr float kInt8Max = 127.0f;
constexpr float kInt8Least = 0x1p-126f;

// append: NormAppendArgs with int8 pools; a.steps: heads of a workgroup (set by the launcher)
hipError_t launch_int8_append(const NormAppendArgs& a, const Int8Scales& s, const AxesArgs* axes, hipStream_t stream);
// workgroups of the append at most, for the host's launch-size check
inline int64_t int8_append_units(const PackedSeqs& s) {
  // a sequence of n tokens falls into at most (n - 1) / 16 + 2 pages, and into no more than n
  const int64_t most = s.n_tokens / kPage + 2 * (int64_t)(s.batch < s.n_tokens ? s.batch : s.n_tokens);
  return most < s.n_tokens ? most : s.n_tokens;
}

// dimensions of the values that a workgroup of a split tile launch sums
constexpr int int8_split_values(int D) { return D == 256 ? 128 : D; }
// attention: PackedAttnArgs with int8 pools (launch_packed_tiles, launch_packed_few for int8 caches)
hipError_t launch_int8_tiles(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream);
hipError_t launch_int8_few(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream);

// the scales of a block: payload [n_layers][2][n_block_pages][Hkv], from (graft) or to (deposit) the pages' ones
struct Int8ScaleCopyArgs {
  Int8Scales scales;
  int64_t n_pages;
  const int32_t* block_table;
  float* payload;
  int32_t first_page, n_block_pages, n_layers, Hkv;
};
__host__ __device__ inline int64_t int8_scale_values(const Int8ScaleCopyArgs& a) { return (int64_t)a.n_layers * 2 * a.n_block_pages * a.Hkv; }
hipError_t launch_int8_scales(const Int8ScaleCopyArgs& a, bool deposit, hipStream_t stream);

}  // namespace kvg
