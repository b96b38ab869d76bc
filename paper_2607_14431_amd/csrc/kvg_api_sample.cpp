// C ABI of sampling (declarations and contracts in include/kvg.h).
#include <hip/hip_runtime.h>

#include "kvg.h"
#include "kvg_host.h"
#include "kvg_sample.h"

namespace {

using namespace kvg::host;

int ceil_log2(int32_t n) {
  int b = 0;
  while (((int64_t)1 << b) < n) ++b;
  return b;
}

}  // namespace

extern "C" {

size_t kvg_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab <= 0 || vocab > (1 << kvg::kSampleIndexBits) || rows > kvg::kMaxSampleRows) return 0;
  return kAlign;
}

int kvg_sample(const float* logits, int64_t row_stride, int32_t rows, int32_t vocab, const kvg_sampling* sampling,
               const double* uniform, int32_t* tokens, float* logprobs, void* ws, size_t ws_bytes, void* stream) {
  if (rows < 0 || vocab <= 0 || sampling == nullptr) return KVG_E_INVAL;
  if (row_stride == 0) row_stride = vocab;
  if (row_stride < vocab) return KVG_E_INVAL;
  if (vocab > (1 << kvg::kSampleIndexBits) || rows > kvg::kMaxSampleRows) return KVG_E_SHAPE;
  if (ws == nullptr || ws_bytes < kvg_sample_workspace_bytes(rows, vocab)) return KVG_E_WORKSPACE;
  if (rows == 0) return KVG_OK;
  if (logits == nullptr || uniform == nullptr || tokens == nullptr || sampling->temperature == nullptr) return KVG_E_INVAL;
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return KVG_E_ALIGN;
  kvg::SampleArgs a;
  a.logits = logits;
  a.row_stride = row_stride;
  a.rows = rows;
  a.V = vocab;
  a.temperature = sampling->temperature;
  a.top_k = sampling->top_k;
  a.top_p = sampling->top_p;
  a.min_p = sampling->min_p;
  a.uniform = uniform;
  a.tokens = tokens;
  a.logprobs = logprobs;
  a.bits = 62 - ceil_log2(vocab);
  return hip_status(kvg::launch_sample(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
