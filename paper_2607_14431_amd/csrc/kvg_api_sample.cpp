// C ABI of sampling (declarations and contracts in include/kvg.h).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvg.h"
#include "kvg_host.h"
#include "kvg_sample.h"

namespace {

using namespace kvg::host;

// Workspace of a call: the arrays of SampleArgs, one after the other.
struct Layout {
  int part_size, n_parts;
  size_t tops, sums, bin_weights, bin_counts, n_listed, listed, total;
};
Layout layout(int64_t rows, int32_t vocab) {
  Layout w = {0, 0, 0, 0, 0, 0, 0, 0, kAlign};
  if (vocab <= kvg::kSampleListed) return w;
  w.part_size = kvg::sample_part_size(rows, vocab);
  w.n_parts = (vocab + w.part_size - 1) / w.part_size;
  w.tops = align_up((size_t)rows * w.n_parts * 8);
  w.sums = w.tops;
  w.bin_weights = align_up((size_t)rows * kvg::kSampleBins * 8);
  w.bin_counts = align_up((size_t)rows * kvg::kSampleBins * 4);
  w.n_listed = align_up((size_t)rows * 4);
  w.listed = align_up((size_t)rows * kvg::kSampleListed * 8);
  w.total = w.tops + w.sums + w.bin_weights + w.bin_counts + w.n_listed + w.listed;
  return w;
}

int ceil_log2(int32_t n) {
  int b = 0;
  while (((int64_t)1 << b) < n) ++b;
  return b;
}

}  // namespace

extern "C" {

size_t kvg_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab <= 0 || vocab > (1 << kvg::kSampleIndexBits) || rows > kvg::kMaxSampleRows) return 0;
  return std::max(layout(rows, vocab).total, kAlign);
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
  const Layout w = layout(rows, vocab);
  a.part_size = w.part_size;
  a.n_parts = w.n_parts;
  char* at = static_cast<char*>(ws);
  auto take = [&](size_t bytes) {
    char* p = at;
    at += bytes;
    return p;
  };
  a.tops = reinterpret_cast<unsigned long long*>(take(w.tops));
  a.sums = reinterpret_cast<unsigned long long*>(take(w.sums));
  a.bin_weights = reinterpret_cast<unsigned long long*>(take(w.bin_weights));
  a.bin_counts = reinterpret_cast<uint32_t*>(take(w.bin_counts));
  a.n_listed = reinterpret_cast<uint32_t*>(take(w.n_listed));
  a.listed = reinterpret_cast<unsigned long long*>(take(w.listed));
  return hip_status(kvg::launch_sample(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
