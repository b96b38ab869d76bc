// Tokens from logits: temperature, top-k, top-p, min-p and given random numbers.
//
// With x_i = (l_i - max l) / T in fp64 a token weighs e^x_i, rounded to fixed point with `bits` bits after the point: sums of a
// row's weights are integers below 2^62, so they have no order and no rounding.  Tokens are ordered by a
// code of 56 bits, the logit's (32 bits that compare as the floats do) over the inverted index: the likelier first, of equal
// ones the lower index.  Each limit keeps a prefix of that order: top-k ends at the k-th largest code, top-p where the running sum
// of weights reaches its share, min-p at a weight.  So what is kept is `code >= cut && e^x >= min_p`, and the token is the first in
// index order whose running sum of kept weights passes the random number's.
//
// A workgroup takes a row.  A cut is found digit by digit (11, 11, 10 bits of the logit, twice 12 of the index): count and weight
// of the tokens that share the digits so far, by their next digit.
#include "kvg_exp.h"
#include "kvg_sample.h"

#include <math.h>

namespace kvg {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 4096;
typedef unsigned long long u64;

constexpr uint32_t kIndexMask = (1u << kSampleIndexBits) - 1;
// Bits that compare as floats do; NaN above all others, -0 as 0.
__device__ __forceinline__ uint32_t logit_code(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return x != x ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t code) { return __uint_as_float(code & 0x80000000u ? code & 0x7FFFFFFFu : ~code); }
__device__ __forceinline__ u64 token_code(float x, int i) { return (u64)logit_code(x) << kSampleIndexBits | (kIndexMask - (uint32_t)i); }
__device__ __forceinline__ int token_of(u64 code) { return (int)(kIndexMask - (uint32_t)(code & kIndexMask)); }

__device__ __forceinline__ u64 add_lanes(u64 x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m);
  return x;
}
__device__ __forceinline__ u64 max_lanes(u64 x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    const u64 y = __shfl_xor(x, m);
    x = y > x ? y : x;
  }
  return x;
}

// A row's parameters.
struct Row {
  double top, inv_t, min_p, one;      // largest logit, 1 / temperature, least e^x kept, 2^bits
  u64 cut;                            // least code kept
};
struct Weight {
  double e;
  u64 n;
};
__device__ __forceinline__ Weight weight(const Row& r, float l, const double* tab) {
  const double e = exp_table(((double)l - r.top) * r.inv_t, tab);
  return {e, (u64)(int64_t)__builtin_rint(e * r.one)};
}
// the weight that a token keeps
__device__ __forceinline__ u64 kept(const Row& r, float l, int i, const double* tab) {
  if (token_code(l, i) < r.cut) return 0;
  const Weight w = weight(r, l, tab);
  return w.e >= r.min_p ? w.n : 0;
}

struct Shared {
  double tab[64];
  u64 wave[kWaves];
  u64 weight[kBins];
  uint32_t count[kBins];
  u64 found[3];
};

// The code at which the running count (or, by_weight, the running weight) of the tokens from the largest code on reaches `need`, of
// those with codes of at least r.cut; there are that many.
__device__ u64 find_cut(const SampleArgs& a, const Row& r, const float* l, bool by_weight, u64 need, Shared& s) {
  constexpr int kShift[5] = {45, 34, 24, 12, 0}, kWidth[5] = {11, 11, 10, 12, 12};
  u64 prefix = 0;
  for (int d = 0; d < 5; ++d) {
    const int n = 1 << kWidth[d], above = kShift[d] + kWidth[d];
    for (int i = threadIdx.x; i < n; i += kThreads) {
      s.count[i] = 0;
      s.weight[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
      const u64 c = token_code(l[i], i);
      if (c < r.cut || c >> above != prefix >> above) continue;
      const int bin = (int)(c >> kShift[d]) & (n - 1);
      if (by_weight)
        atomicAdd(&s.weight[bin], weight(r, l[i], s.tab).n);
      else
        atomicAdd(&s.count[bin], 1u);
    }
    __syncthreads();
    // the highest bins first: lane j of the first wave sums n / 64 of them, then finds the one that reaches `need`
    if (threadIdx.x < 64) {
      const int per = n / 64, hi = n - 1 - (int)threadIdx.x * per;
      u64 sum = 0;
      for (int j = 0; j < per; ++j) sum += by_weight ? s.weight[hi - j] : s.count[hi - j];
      u64 upto = sum;
      for (int m = 1; m < 64; m <<= 1) {
        const u64 before = __shfl_up(upto, m);
        upto += (int)threadIdx.x >= m ? before : 0;
      }
      const uint64_t reach = __builtin_amdgcn_ballot_w64(upto >= need);
      if (reach != 0 && (int)threadIdx.x == __builtin_ctzll(reach)) {
        u64 run = upto - sum;
        for (int j = 0; j < per; ++j) {
          const u64 x = by_weight ? s.weight[hi - j] : s.count[hi - j];
          if (run + x >= need) {
            s.found[0] = (u64)(hi - j);
            s.found[1] = run;
            break;
          }
          run += x;
        }
      }
    }
    __syncthreads();
    prefix |= s.found[0] << kShift[d];
    need -= s.found[1];
    __syncthreads();
  }
  return prefix;
}

// Weight kept in [i0, i1), each wave a part of it: s.wave[w] is that of [i0 + w part, i0 + (w + 1) part).  The sum.
__device__ u64 part_weights(const Row& r, const float* l, int i0, int i1, int part, Shared& s) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  u64 sum = 0;
  const int end = min(i1, i0 + (wave + 1) * part);
  for (int i = i0 + wave * part + lane; i < end; i += 64) sum += kept(r, l[i], i, s.tab);
  sum = add_lanes(sum);
  __syncthreads();
  if (lane == 0) s.wave[wave] = sum;
  __syncthreads();
  u64 total = 0;
  for (int w = 0; w < kWaves; ++w) total += s.wave[w];
  return total;
}

__global__ __launch_bounds__(kThreads) void sample_row_kernel(const SampleArgs a) {
  __shared__ Shared s;
  const int row = blockIdx.x, tid = threadIdx.x;
  const float* l = a.logits + (int64_t)row * a.row_stride;
  if (tid < 64) s.tab[tid] = exp2(tid / 64.0);
  u64 top = 0;
  for (int i = tid; i < a.V; i += kThreads) {
    const u64 c = token_code(l[i], i);
    top = c > top ? c : top;
  }
  top = max_lanes(top);
  if ((tid & 63) == 0) s.wave[tid >> 6] = top;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) top = s.wave[w] > top ? s.wave[w] : top;
  __syncthreads();

  const float t = a.temperature[row];
  const double u = a.uniform[row];
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.0f;
  const float m = a.min_p != nullptr ? a.min_p[row] : 0.0f;
  Row r;
  const uint32_t top_code = (uint32_t)(top >> kSampleIndexBits);
  r.top = logit_of(top_code);
  const bool ok = top_code < logit_code(INFINITY) && top_code > logit_code(-INFINITY) && t >= 0.0f && t < INFINITY && u == u && p == p && m == m;
  if (!ok || t == 0.0f) {
    if (tid == 0) {
      a.tokens[row] = ok ? token_of(top) : -1;
      if (a.logprobs != nullptr) a.logprobs[row] = ok ? 0.0f : __uint_as_float(0x7FC00000u);
    }
    return;
  }
  r.inv_t = 1.0 / (double)t;
  r.min_p = m < 1.0f ? m : 1.0;
  r.one = __builtin_ldexp(1.0, a.bits);
  r.cut = 0;
  if (k > 0 && k < a.V) r.cut = find_cut(a, r, l, false, (u64)k, s);
  const int part = (a.V + kWaves - 1) / kWaves;
  if (p < 1.0f) {
    Row all = r;
    all.min_p = 0.0;
    const u64 sum = part_weights(all, l, 0, a.V, part, s);
    u64 need = p > 0.0f ? (u64)(int64_t)__builtin_ceil((double)p * (double)sum) : 1;
    need = need < 1 ? 1 : need > sum ? sum : need;
    r.cut = find_cut(a, r, l, true, need, s);
  }
  const u64 total = part_weights(r, l, 0, a.V, part, s);
  u64 target = u > 0.0 ? (u < 1.0 ? (u64)(int64_t)__builtin_floor(u * (double)total) : total - 1) : 0;
  target = target < total ? target : total - 1;
  // the part that holds it, ever shorter
  int i0 = 0, i1 = a.V, size = part;
  while (true) {
    int w = 0;
    while (w < kWaves - 1 && target >= s.wave[w]) target -= s.wave[w++];
    i0 += w * size;
    i1 = min(i1, i0 + size);
    if (size <= 64) break;
    size = (size + kWaves - 1) / kWaves;
    __syncthreads();
    part_weights(r, l, i0, i1, size, s);
  }
  // at most 64 tokens are left: a lane each
  if (tid >= 64) return;
  const int i = i0 + tid;
  u64 upto = i < i1 ? kept(r, l[i], i, s.tab) : 0;
  for (int d = 1; d < 64; d <<= 1) {
    const u64 before = __shfl_up(upto, d);
    upto += tid >= d ? before : 0;
  }
  const uint64_t past = __builtin_amdgcn_ballot_w64(upto > target);
  if (past != 0 && tid == __builtin_ctzll(past)) {
    a.tokens[row] = i;
    if (a.logprobs != nullptr)
      a.logprobs[row] = (float)(((double)l[i] - r.top) * r.inv_t - (log((double)total) - a.bits * 0.69314718055994530942));
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
  sample_row_kernel<<<a.rows, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace kvg
