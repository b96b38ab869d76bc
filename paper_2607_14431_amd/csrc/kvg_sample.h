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
// Codes that a workgroup sorts.
constexpr int kSampleListed = 4096;

// Parts of a row: enough to spread few rows over the chip, multiples of 1,024 tokens.
constexpr int kSampleParts = 128;
inline int sample_part_size(int64_t rows, int64_t V) {
  const int64_t want = rows < 16 ? kSampleParts : rows < 1024 ? 2048 / rows : 2;
  return (int)(((V + want - 1) / want + 1023) / 1024 * 1024);
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream);

}  // namespace kvg
