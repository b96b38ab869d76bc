// Sampling: kernel parameter block and launcher.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvg {

constexpr int kMaxSampleRows = 65535;
constexpr int kSampleIndexBits = 24;      // vocabularies of up to 2^24 tokens

struct SampleArgs {
  const float* logits;
  int64_t row_stride;
  int32_t rows, V;
  const float* temperature;
  const int32_t* top_k;       // or null, as the next two
  const float* top_p;
  const float* min_p;
  const double* uniform;
  int32_t* tokens;
  float* logprobs;            // or null
  int32_t bits;               // after the point of a weight: 62 - ceil(log2 V)
  // Longer rows than kSampleListed: cut into n_parts parts of part_size tokens, and in the workspace, of every row,
  int32_t n_parts, part_size;
  unsigned long long* tops;          // [n_parts] largest code of a part
  unsigned long long* sums;          // [n_parts] weight of a part's tokens that are kept whatever the list says
  unsigned long long* bin_weights;   // [kSampleBins] weight and number of the tokens of a bin
  uint32_t* bin_counts;
  uint32_t* n_listed;                // length of the list and the list, of the codes between which a limit's end lies
  unsigned long long* listed;        // [kSampleListed]
};

// Bins of a row's tokens by their weight, the heaviest first.
constexpr int kSampleBins = 1024;
// Codes that a workgroup holds.
constexpr int kSampleListed = 4096;

// Parts of a row, multiples of 1,024 tokens: few rows need many to spread over the chip, of more each part's workgroup should have
// more than its start to do.  Rows of 262,144 tokens with top-k, top-p and min-p, us, 128 parts / 64 / 32 / 8: 1 row 28.3 / 27.7 / 32.4 / 52, 16 rows
// 44 / 40 / 42 / 70, 64 rows 92 / 74 / 68 / 81, 256 rows 276 / 195 / 172 / 173.  Of 32,000 tokens, parts of 1,024 / 2,048 / 4,096 / 8,192: 1 row 25.0 /
// 25.5 / 27.1 / 32.2, 16 rows 31 / 30 / 30 / 35, 64 rows 42 / 36 / 34 / 38, 256 rows 82 / 59 / 48 / 49.
constexpr int kSampleParts = 128;
inline int sample_part_size(int64_t rows, int64_t V) {
  const int64_t want = rows < 16 ? kSampleParts : rows < 32 ? 64 : 32, least = rows < 16 ? 1024 : 4096;
  return (int)(((V + want - 1) / want + least - 1) / least * least);
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream);

}  // namespace kvg
