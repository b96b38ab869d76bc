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
};

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream);

}  // namespace kvg
