// Tokens from logits: temperature, top-k, top-p, min-p and given random numbers.
//
// With x_i = (l_i - max l) / T in fp64 a token weighs e^x_i, rounded to fixed point with `bits` bits after the point: sums of a
// row's weights are integers below 2^62, so they have no order and no rounding.  Tokens are ordered by a
// code of 56 bits, the logit's (32 bits that compare as the floats do) over the inverted index: the likelier first, of equal
// ones the lower index.  Each limit keeps a prefix of that order: top-k ends at the k-th largest code, top-p where the running sum
// of weights reaches its share, min-p at a weight.  So what is kept is `code >= cut && e^x >= min_p`, and the token is the first in
// index order whose running sum of kept weights passes the random number's.
//
// Rows of up to kSampleListed tokens: a workgroup sorts the row's codes.  Longer ones in passes over the row, by many workgroups:
//   top     the largest logit of every part of the row
//   bins    count and weight of the row's tokens by weight (1,024 equal steps of the exponent down to weight 0), where a top-k or
//           top-p may end inside the row.  The bins tell in which of them the two limits end.  Weights are left out where top-p is 1
//           or the tokens of top-k are few (by_list): an exponential in fp64 costs more than all else in the pass
//   parts   the weight of every part's tokens in the bins before those, and a list of the codes in them
//   pick    a workgroup a row: the list, sorted, gives the cut; the parts' weights the part that holds the token, which is searched
// Where the list would be too long (thousands of tokens of nearly equal logits) the cut is found digit by digit instead (11, 11, 10
// bits of the logit, twice 12 of the index): count or weight of the tokens that share the digits so far, by their next digit.
#include "kvg_exp.h"
#include "kvg_sample.h"

#include <math.h>

namespace kvg {

namespace {

constexpr int kThreads = 1024;            // of the workgroup that picks a row's token
constexpr int kPartThreads = 256;         // of one that takes a part of a row
constexpr int kPartListed = 512;          // codes that it lists together
constexpr double kLn2 = 0.69314718055994530942;
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
  float least;                        // logits below it weigh 0
  double bin_scale;                   // bins for each unit of x
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

struct Digits {
  u64 weight[kBins];
  uint32_t count[kBins];
};
struct Shared {
  double tab[64];
  u64 wave[kWaves];
  u64 found[2];
  union {
    Digits digits;
    u64 list[kSampleListed];
  };
};

// The share p of a weight, rounded up: what a running sum has to reach.
__device__ __forceinline__ u64 share_of(float p, u64 sum) {
  const u64 need = p > 0.0f ? (u64)(int64_t)__builtin_ceil((double)p * (double)sum) : 1;
  return need < 1 ? 1 : need > sum && sum > 0 ? sum : need;
}

// The code at which the running count (or, by_weight, the running weight) of the tokens from the largest code on reaches `need`, of
// those with codes of at least r.cut; there are that many.
__device__ u64 find_cut(const SampleArgs& a, const Row& r, const float* l, bool by_weight, u64 need, Shared& s) {
  constexpr int kShift[5] = {45, 34, 24, 12, 0}, kWidth[5] = {11, 11, 10, 12, 12};
  u64 prefix = 0;
  for (int d = 0; d < 5; ++d) {
    const int n = 1 << kWidth[d], above = kShift[d] + kWidth[d];
    for (int i = threadIdx.x; i < n; i += kThreads) {
      s.digits.count[i] = 0;
      s.digits.weight[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
      const u64 c = token_code(l[i], i);
      if (c < r.cut || c >> above != prefix >> above) continue;
      const int bin = (int)(c >> kShift[d]) & (n - 1);
      if (by_weight)
        atomicAdd(&s.digits.weight[bin], weight(r, l[i], s.tab).n);
      else
        atomicAdd(&s.digits.count[bin], 1u);
    }
    __syncthreads();
    // the highest bins first: lane j of the first wave sums n / 64 of them, then finds the one that reaches `need`
    if (threadIdx.x < 64) {
      const int per = n / 64, hi = n - 1 - (int)threadIdx.x * per;
      u64 sum = 0;
      for (int j = 0; j < per; ++j) sum += by_weight ? s.digits.weight[hi - j] : s.digits.count[hi - j];
      u64 upto = sum;
      for (int m = 1; m < 64; m <<= 1) {
        const u64 before = __shfl_up(upto, m);
        upto += (int)threadIdx.x >= m ? before : 0;
      }
      const uint64_t reach = __builtin_amdgcn_ballot_w64(upto >= need);
      if (reach != 0 && (int)threadIdx.x == __builtin_ctzll(reach)) {
        u64 run = upto - sum;
        for (int j = 0; j < per; ++j) {
          const u64 x = by_weight ? s.digits.weight[hi - j] : s.digits.count[hi - j];
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

// A row's parameters from its largest code; false where the row has no token to sample, or takes its first maximum: what it gives is
// then written (by one lane).
__device__ __forceinline__ bool row_setup(const SampleArgs& a, int row, u64 top, bool write, Row& r) {
  const float t = a.temperature[row];
  const double u = a.uniform[row];
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.0f;
  const float m = a.min_p != nullptr ? a.min_p[row] : 0.0f;
  const uint32_t top_code = (uint32_t)(top >> kSampleIndexBits);
  const bool ok = top_code < logit_code(INFINITY) && top_code > logit_code(-INFINITY) && t >= 0.0f && t < INFINITY && u == u && p == p && m == m;
  if (!ok || t == 0.0f) {
    if (write) {
      a.tokens[row] = ok ? token_of(top) : -1;
      if (a.logprobs != nullptr) a.logprobs[row] = ok ? 0.0f : __uint_as_float(0x7FC00000u);
    }
    return false;
  }
  r.top = logit_of(top_code);
  r.inv_t = 1.0 / (double)t;
  r.min_p = m < 1.0f ? m : 1.0;
  r.one = __builtin_ldexp(1.0, a.bits);
  r.cut = 0;
  // weights below half of 2^-bits are 0: no logit further below the top than (bits + 1) ln 2 t has one
  r.least = (float)(r.top - (a.bits + 2) * kLn2 * (double)t) ;
  r.least = r.least - fabsf(r.least) * 0x1p-22f - 1e-37f;
  r.bin_scale = kSampleBins / ((a.bits + 2) * kLn2);
  return true;
}
__device__ __forceinline__ int bin_of(const Row& r, float l) {
  const double b = (r.top - (double)l) * r.inv_t * r.bin_scale;
  return b < kSampleBins - 1 ? (int)b : kSampleBins - 1;
}

// f(logit, index) for the tokens [i0, i1) of a row, by `threads` lanes; four at a time where the row lies on 16 bytes (i0 is a
// multiple of 4)
template <typename F>
__device__ __forceinline__ void for_tokens(const float* l, int i0, int i1, int threads, F f) {
  if (reinterpret_cast<uintptr_t>(l) % 16 == 0) {
    int i = i0 + 4 * (int)threadIdx.x;
#pragma unroll 2
    for (; i + 3 < i1; i += 4 * threads) {
      const float4 x = *reinterpret_cast<const float4*>(l + i);
      f(x.x, i);
      f(x.y, i + 1);
      f(x.z, i + 2);
      f(x.w, i + 3);
    }
    for (; i < i1; ++i) f(l[i], i);      // the lane whose four reach past the end
  } else {
    for (int i = i0 + (int)threadIdx.x; i < i1; i += threads) f(l[i], i);
  }
}

// The largest code of a row's parts.
__device__ __forceinline__ u64 row_top(const SampleArgs& a, int row) {
  u64 top = 0;
  for (int i = threadIdx.x & 63; i < a.n_parts; i += 64) {
    const u64 c = a.tops[(int64_t)row * a.n_parts + i];
    top = c > top ? c : top;
  }
  return max_lanes(top);
}

__global__ __launch_bounds__(kPartThreads) void sample_top_kernel(const SampleArgs a) {
  __shared__ u64 sh[kPartThreads / 64];
  const int row = blockIdx.y, part = blockIdx.x;
  const float* l = a.logits + (int64_t)row * a.row_stride;
  // the row's bins and list, emptied for the next launches
  for (int i = part * kPartThreads + threadIdx.x; i < kSampleBins; i += a.n_parts * kPartThreads) {
    a.bin_weights[(int64_t)row * kSampleBins + i] = 0;
    a.bin_counts[(int64_t)row * kSampleBins + i] = 0;
  }
  if (part == 0 && threadIdx.x == 0) a.n_listed[row] = 0;
  u64 top = 0;
  for_tokens(l, part * a.part_size, min(a.V, (part + 1) * a.part_size), kPartThreads, [&](float x, int i) {
    const u64 c = token_code(x, i);
    top = c > top ? c : top;
  });
  top = max_lanes(top);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kPartThreads / 64; ++w) top = sh[w] > top ? sh[w] : top;
  a.tops[(int64_t)row * a.n_parts + part] = top;
}

// Whether top-k's tokens are few enough that all of them are listed and top-p's end is sought in the list.
__device__ __forceinline__ bool by_list(const SampleArgs& a, int row) {
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  return k > 0 && k <= kSampleListed / 4;
}
__device__ __forceinline__ bool has_top_p(const SampleArgs& a, int row) { return a.top_p != nullptr && a.top_p[row] < 1.0f; }
// Whether a row's top-k or top-p may end inside it.
__device__ __forceinline__ bool limited(const SampleArgs& a, int row) {
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  return (k > 0 && k < a.V) || has_top_p(a, row);
}

__global__ __launch_bounds__(kPartThreads) void sample_bins_kernel(const SampleArgs a) {
  __shared__ double tab[64];
  __shared__ u64 weights[kSampleBins];
  __shared__ uint32_t counts[kSampleBins];
  const int row = blockIdx.y, part = blockIdx.x;
  Row r;
  if (!limited(a, row) || !row_setup(a, row, row_top(a, row), false, r)) return;
  if (threadIdx.x < 64) tab[threadIdx.x] = exp2(threadIdx.x / 64.0);
  for (int i = threadIdx.x; i < kSampleBins; i += kPartThreads) {
    weights[i] = 0;
    counts[i] = 0;
  }
  __syncthreads();
  const float* l = a.logits + (int64_t)row * a.row_stride;
  const int i0 = part * a.part_size, i1 = min(a.V, i0 + a.part_size);
  const bool weigh = has_top_p(a, row) && !by_list(a, row);
  if (weigh)
    for_tokens(l, i0, i1, kPartThreads, [&](float x, int) {
      if (x < r.least) return;
      const int b = bin_of(r, x);
      atomicAdd(&weights[b], weight(r, x, tab).n);
      atomicAdd(&counts[b], 1u);
    });
  else
    for_tokens(l, i0, i1, kPartThreads, [&](float x, int) {
      if (x >= r.least) atomicAdd(&counts[bin_of(r, x)], 1u);
    });
  __syncthreads();
  for (int i = threadIdx.x; i < kSampleBins; i += kPartThreads)
    if (counts[i] != 0) {
      if (weigh) atomicAdd(&a.bin_weights[(int64_t)row * kSampleBins + i], weights[i]);
      atomicAdd(&a.bin_counts[(int64_t)row * kSampleBins + i], counts[i]);
    }
}

// Where a row's limits end, from its bins.
struct Ends {
  int first, last;            // bins between which top-p ends (top-k's, where there is no top-p; all from the first one on by_list):
                              // all before `first` is kept
  int k_bin;                  // the bin that top-k ends in, kSampleBins: none
  uint32_t k_need;            // tokens that top-k takes of it
  uint32_t listed_before_k;   // of the listed codes, those in bins before k_bin
  u64 before_first, before_k; // weight of the bins before
};
struct EndsShared {
  u64 weight[16], count[16];  // of the waves' bins
  u64 upto_k;                 // weight up to top-k's bin, with it
  Ends ends;
};
// (all lanes of a workgroup of kSampleBins lanes or fewer; bins in order, kSampleBins / threads a lane)
template <int kT>
__device__ void find_ends(const SampleArgs& a, int row, Ends& out, EndsShared& s) {
  constexpr int kPer = kSampleBins / kT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = threadIdx.x * kPer;
  u64 w[kPer], c[kPer], sw = 0, sc = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    w[i] = a.bin_weights[(int64_t)row * kSampleBins + b0 + i];
    c[i] = a.bin_counts[(int64_t)row * kSampleBins + b0 + i];
    sw += w[i];
    sc += c[i];
  }
  u64 uw = sw, uc = sc;                                      // up to and with this lane's
  for (int m = 1; m < 64; m <<= 1) {
    const u64 x = __shfl_up(uw, m), y = __shfl_up(uc, m);
    uw += lane >= m ? x : 0;
    uc += lane >= m ? y : 0;
  }
  if (lane == 63) {
    s.weight[wave] = uw;
    s.count[wave] = uc;
  }
  if (threadIdx.x == 0) s.ends = {0, -1, kSampleBins, 0, 0, 0, 0};
  __syncthreads();
  u64 total_w = 0, total_c = 0;
  for (int i = 0; i < kT / 64; ++i) {
    if (i < wave) {
      uw += s.weight[i];
      uc += s.count[i];
    }
    total_w += s.weight[i];
    total_c += s.count[i];
  }
  uw -= sw;                                                  // before this lane's
  uc -= sc;
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.0f;
  const bool by_k = k > 0 && (u64)k < total_c;
  if (by_k) {
    u64 x = uw, y = uc;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (y < (u64)k && y + c[i] >= (u64)k) {
        s.ends.k_bin = b0 + i;
        s.ends.k_need = (uint32_t)((u64)k - y);
        s.ends.before_k = x;
        s.upto_k = x + w[i];
      }
      x += w[i];
      y += c[i];
    }
  }
  __syncthreads();
  const u64 most = by_k ? s.upto_k : total_w, least = by_k ? s.ends.before_k : total_w;
  if (p < 1.0f && by_list(a, row)) {
    if (threadIdx.x == 0) {
      s.ends.first = 0;
      s.ends.last = by_k ? s.ends.k_bin : kSampleBins - 1;   // all of the row, k or fewer tokens
    }
  } else if (p < 1.0f) {
    const u64 need0 = share_of(p, least), need1 = share_of(p, most);
    u64 x = uw;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (x < need0 && x + w[i] >= need0) {
        s.ends.first = b0 + i;
        s.ends.before_first = x;
      }
      if (x < need1 && x + w[i] >= need1) s.ends.last = b0 + i;
      x += w[i];
    }
  } else if (by_k && threadIdx.x == 0) {
    s.ends.first = s.ends.last = s.ends.k_bin;
    s.ends.before_first = s.ends.before_k;
  } else if (threadIdx.x == 0) {
    s.ends.first = kSampleBins;                              // no limit ends in the row
  }
  __syncthreads();
  if (s.ends.k_bin < kSampleBins) {                          // listed codes in front of top-k's bin
    u64 n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) n += b0 + i >= s.ends.first && b0 + i <= s.ends.last && b0 + i < s.ends.k_bin ? c[i] : 0;
    n = add_lanes(n);
    if (lane == 0 && n != 0) atomicAdd(&s.ends.listed_before_k, (uint32_t)n);
  }
  __syncthreads();
  out = s.ends;
}
__device__ __forceinline__ bool is_listed(const Ends& e, int bin) { return (bin >= e.first && bin <= e.last) || bin == e.k_bin; }

__global__ __launch_bounds__(kPartThreads) void sample_parts_kernel(const SampleArgs a) {
  __shared__ double tab[64];
  __shared__ EndsShared ends_shared;
  __shared__ u64 sh[kPartThreads / 64];
  __shared__ u64 listed[kPartListed];                        // this part's, one reservation of the row's list for all
  __shared__ uint32_t n_here, at_row;
  const int row = blockIdx.y, part = blockIdx.x;
  if (threadIdx.x == 0) n_here = 0;
  Row r;
  if (!row_setup(a, row, row_top(a, row), false, r)) return;
  if (threadIdx.x < 64) tab[threadIdx.x] = exp2(threadIdx.x / 64.0);
  Ends ends = {kSampleBins, -1, kSampleBins, 0, 0, 0, 0};
  if (limited(a, row)) find_ends<kPartThreads>(a, row, ends, ends_shared);
  __syncthreads();
  const bool all = ends.first == kSampleBins;
  // logits below `low` are in later bins, or below min-p where that is the only limit; the rounding of these lines is below its slack
  float low = r.least;
  {
    const int after = (all ? kSampleBins : max(ends.last, ends.k_bin < kSampleBins ? ends.k_bin : 0)) + 1;
    const double span = all ? (r.min_p > 0.0 ? -log(r.min_p) : INFINITY) / r.inv_t : after / (r.inv_t * r.bin_scale);
    if (after < kSampleBins || (all && span < INFINITY)) {
      const float x = (float)(r.top - span);
      low = fmaxf(low, x - (float)((fabs(r.top) + span + 1.0 / r.inv_t) * 0x1p-22) - 1e-37f);
    }
  }
  u64 sum = 0;
  for_tokens(a.logits + (int64_t)row * a.row_stride, part * a.part_size, min(a.V, (part + 1) * a.part_size), kPartThreads, [&](float x, int i) {
    if (x < low) return;
    const int b = all ? 0 : bin_of(r, x);
    if (b < ends.first) {
      const Weight w = weight(r, x, tab);
      sum += w.e >= r.min_p ? w.n : 0;
    } else if (is_listed(ends, b)) {
      const uint32_t at = atomicAdd(&n_here, 1u);
      if (at < kPartListed) {
        listed[at] = token_code(x, i);
      } else {
        const uint32_t far = atomicAdd(&a.n_listed[row], 1u);
        if (far < kSampleListed) a.listed[(int64_t)row * kSampleListed + far] = token_code(x, i);
      }
    }
  });
  sum = add_lanes(sum);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
  __syncthreads();
  const int n = min((int)n_here, kPartListed);
  if (threadIdx.x == 0) {
    for (int w = 1; w < kPartThreads / 64; ++w) sum += sh[w];
    a.sums[(int64_t)row * a.n_parts + part] = sum;
    if (n > 0) at_row = atomicAdd(&a.n_listed[row], (uint32_t)n);
  }
  if (n == 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPartThreads)
    if (at_row + i < kSampleListed) a.listed[(int64_t)row * kSampleListed + at_row + i] = listed[i];
}

// The larger (or smaller) of a code and the one that `d` places away.
__device__ __forceinline__ u64 keep(u64 x, u64 y, bool larger) { return (x > y) == larger ? x : y; }

// Sorts the n codes of a list, the largest first, `size` a power of two with zeros behind them, kPer consecutive ones a lane: pairs
// within a lane or a wave meet in registers, others in the list.  (all lanes)
template <int kPer>
__device__ void sort_codes(u64* list, int n, int size) {
  const int at = threadIdx.x * kPer;
  u64 x[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) x[j] = at + j < n ? list[at + j] : 0;
  for (int run = 2; run <= size; run <<= 1)
    for (int d = run >> 1; d > 0; d >>= 1) {
      // whether this lane's lower code of a pair is the larger one, and whether it has the lower ones (d and run of kPer or more)
      if (d >= 64 * kPer) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (at < size) list[at + j] = x[j];
        __syncthreads();
        if (at < size) {
#pragma unroll
          for (int j = 0; j < kPer; ++j) x[j] = keep(x[j], list[(at + j) ^ d], ((at & d) == 0) == ((at & run) == 0));
        }
      } else if (d >= kPer) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[j] = keep(x[j], __shfl_xor(x[j], d / kPer), ((at & d) == 0) == ((at & run) == 0));
      } else {
#pragma unroll
        for (int e = 1; e < kPer; e <<= 1)
          if (d == e) {
            u64 y[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) y[j] = keep(x[j], x[j ^ e], ((j & e) == 0) == (((at + j) & run) == 0));
#pragma unroll
            for (int j = 0; j < kPer; ++j) x[j] = y[j];
          }
      }
    }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (at + j < n) list[at + j] = x[j];
  __syncthreads();
}
// (all lanes; the list is written)
__device__ void sort_list(u64* list, int n) {
  int size = 64;
  while (size < n) size <<= 1;
  if (size <= kThreads)
    sort_codes<1>(list, n, size);
  else
    sort_codes<kSampleListed / kThreads>(list, n, size);
}

// The first place of a sorted list, of n, at which `base` and the weights up to it reach `need`; n - 1 if none.  (all lanes)
__device__ int reach(const Row& r, const u64* list, int n, u64 base, u64 need, Shared& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (n + kThreads - 1) / kThreads, j0 = threadIdx.x * per;
  u64 sum = 0;
  for (int j = j0; j < min(n, j0 + per); ++j) sum += weight(r, logit_of((uint32_t)(list[j] >> kSampleIndexBits)), s.tab).n;
  u64 upto = sum;
  for (int m = 1; m < 64; m <<= 1) {
    const u64 x = __shfl_up(upto, m);
    upto += lane >= m ? x : 0;
  }
  __syncthreads();
  if (lane == 63) s.wave[wave] = upto;
  if (threadIdx.x == 0) s.found[0] = (u64)(n - 1);
  __syncthreads();
  u64 run = base + upto - sum;
  for (int w = 0; w < wave; ++w) run += s.wave[w];
  if (run < need)
    for (int j = j0; j < min(n, j0 + per); ++j) {
      run += weight(r, logit_of((uint32_t)(list[j] >> kSampleIndexBits)), s.tab).n;
      if (run >= need) {
        s.found[0] = (u64)j;
        break;
      }
    }
  __syncthreads();
  return (int)s.found[0];
}
// The weight of the first n codes of a list.  (all lanes)
__device__ u64 list_weight(const Row& r, const u64* list, int n, Shared& s) {
  u64 sum = 0;
  for (int j = threadIdx.x; j < n; j += kThreads) sum += weight(r, logit_of((uint32_t)(list[j] >> kSampleIndexBits)), s.tab).n;
  sum = add_lanes(sum);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = sum;
  __syncthreads();
  u64 total = 0;
  for (int w = 0; w < kWaves; ++w) total += s.wave[w];
  return total;
}

// Up to and with each lane's, in order.
__device__ __forceinline__ u64 scan_lanes(u64 x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const u64 before = __shfl_up(x, m);
    x += (int)(threadIdx.x & 63) >= m ? before : 0;
  }
  return x;
}

// Up to 64 listed codes, one a lane: the largest first.
__device__ __forceinline__ u64 sort_lanes(u64 c, int n) {
  const int lane = threadIdx.x & 63;
  int rank = 0;
  for (int j = 0; j < n; ++j) {                              // n is the wave's
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)c, j), hi = __builtin_amdgcn_readlane((int)(uint32_t)(c >> 32), j);
    rank += ((u64)hi << 32 | lo) > c;
  }
  const int to = 4 * (lane < n ? rank : lane);
  const uint32_t lo = __builtin_amdgcn_ds_permute(to, (int)(uint32_t)c), hi = __builtin_amdgcn_ds_permute(to, (int)(uint32_t)(c >> 32));
  return (u64)hi << 32 | lo;
}

// kListed: rows of up to kSampleListed tokens, all of them listed.
template <bool kListed>
__global__ __launch_bounds__(kThreads) void sample_pick_kernel(const SampleArgs a) {
  __shared__ Shared s;
  __shared__ EndsShared ends_shared;
  __shared__ u64 parts[kSampleParts];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const float* l = a.logits + (int64_t)row * a.row_stride;
  if (tid < 64) s.tab[tid] = exp2(tid / 64.0);
  u64 top = 0, early = 0;                                    // early: the first listed codes, every wave alike
  uint32_t n_listed = 0;
  if constexpr (kListed) {
    for (int i = tid; i < a.V; i += kThreads) {
      const u64 c = s.list[i] = token_code(l[i], i);
      top = c > top ? c : top;
    }
    top = max_lanes(top);
    if (lane == 0) s.wave[tid >> 6] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = s.wave[w] > top ? s.wave[w] : top;
    __syncthreads();
  } else {
    n_listed = __builtin_amdgcn_readfirstlane((int)a.n_listed[row]);
    early = a.listed[(int64_t)row * kSampleListed + lane];
    for (int i = tid; i < a.n_parts; i += kThreads) parts[i] = a.sums[(int64_t)row * a.n_parts + i];
    top = row_top(a, row);
  }
  Row r;
  if (!row_setup(a, row, top, tid == 0, r)) return;
  const double u = a.uniform[row];
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.0f;
  __syncthreads();
  const bool limit = limited(a, row);
  bool searched = false;                                     // by parts of the row
  if constexpr (kListed) {
    if (limit) {
      sort_list(s.list, a.V);
      int n = k > 0 && k < a.V ? k : a.V;
      if (p < 1.0f) n = reach(r, s.list, n, 0, share_of(p, list_weight(r, s.list, n, s)), s) + 1;
      r.cut = s.list[n - 1];
      __syncthreads();
    }
  } else {
    Ends ends = {kSampleBins, -1, kSampleBins, 0, 0, 0, 0};
    if (limit) find_ends<kThreads>(a, row, ends, ends_shared);
    searched = !limit || n_listed <= kSampleListed;
    if (!searched) {
      if (k > 0 && k < a.V) r.cut = find_cut(a, r, l, false, (u64)k, s);
      if (p < 1.0f) {
        Row whole = r;
        whole.min_p = 0.0;
        r.cut = find_cut(a, r, l, true, share_of(p, part_weights(whole, l, 0, a.V, (a.V + kWaves - 1) / kWaves, s)), s);
      }
    } else if (ends.first < kSampleBins) {
      // n: listed tokens of top-k; `from` on, their weight is added to `base`, and gives what top-p has a share of
      const bool by_k = ends.k_bin < kSampleBins, whole = by_list(a, row);
      int n = by_k ? (int)(ends.listed_before_k + ends.k_need) : (int)n_listed;
      const int from = by_k && !whole ? (int)ends.listed_before_k : 0;
      u64 base = by_k ? ends.before_k : 0;
      if (!by_k && !whole)
        for (int i = 0; i < kWaves; ++i) base += ends_shared.weight[i];
      const bool add = by_k || whole;
      auto to_part = [&](u64 c) {                            // a listed token that is kept, to its part
        const Weight w = weight(r, logit_of((uint32_t)(c >> kSampleIndexBits)), s.tab);
        if (w.e >= r.min_p) atomicAdd(&parts[token_of(c) / a.part_size], w.n);
      };
      if (n_listed <= 64) {                                  // every wave alike, without a barrier
        const u64 c = sort_lanes(lane < (int)n_listed ? early : 0, (int)n_listed);
        if (p < 1.0f) {
          const u64 upto = scan_lanes(lane < n ? weight(r, logit_of((uint32_t)(c >> kSampleIndexBits)), s.tab).n : 0);
          const u64 before = from > 0 ? __shfl(upto, from - 1) : 0;
          const u64 need = share_of(p, base + (add ? __shfl(upto, n - 1) - before : 0));
          const uint64_t past = __builtin_amdgcn_ballot_w64(lane < n && ends.before_first + upto >= need);
          if (past != 0) n = __builtin_ctzll(past) + 1;
        }
        r.cut = __shfl(c, n - 1);
        if (tid < n) to_part(c);
      } else {
        for (int i = tid; i < (int)n_listed; i += kThreads) s.list[i] = a.listed[(int64_t)row * kSampleListed + i];
        __syncthreads();
        sort_list(s.list, (int)n_listed);
        if (p < 1.0f) {
          if (add) base += list_weight(r, s.list + from, n - from, s);
          n = reach(r, s.list, n, ends.before_first, share_of(p, base), s) + 1;
        }
        r.cut = s.list[n - 1];
        for (int i = tid; i < n; i += kThreads) to_part(s.list[i]);
      }
    }
    __syncthreads();
  }
  // the tokens [i0, i1) hold the one that is picked, `target` of their kept weight before it
  int i0 = 0, i1 = a.V;
  u64 total = 0, target = 0;
  auto set_target = [&]() {
    target = u > 0.0 ? (u < 1.0 ? (u64)(int64_t)__builtin_floor(u * (double)total) : total - 1) : 0;
    target = target < total ? target : total - 1;
  };
  if (searched) {
    static_assert(kSampleParts == 128, "two parts a lane");
    const int pair = 2 * lane;                               // every wave alike: a lane's parts, and those up to them
    const u64 even = pair < a.n_parts ? parts[pair] : 0, odd = pair + 1 < a.n_parts ? parts[pair + 1] : 0;
    const u64 upto = scan_lanes(even + odd);
    total = __shfl(upto, 63);
    set_target();
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > target));
    target -= __shfl(upto - odd - even, at);
    const u64 first = __shfl(even, at);
    const bool second = target >= first;
    target -= second ? first : 0;
    i0 = (2 * at + second) * a.part_size;
    i1 = min(a.V, i0 + a.part_size);
  }
  constexpr int kPer = 4;                                    // tokens of a lane in the end
  for (bool first = !kListed && !searched; i1 - i0 > kPer * kThreads; first = false) {
    const int size = (i1 - i0 + kWaves - 1) / kWaves;
    const u64 sum = part_weights(r, l, i0, i1, size, s);
    if (first) {
      total = sum;
      set_target();
    }
    int w = 0;
    while (w < kWaves - 1 && target >= s.wave[w]) target -= s.wave[w++];
    i0 += w * size;
    i1 = min(i1, i0 + size);
  }
  // a few consecutive tokens a lane
  const int per = (i1 - i0 + kThreads - 1) / kThreads;
  u64 mine[kPer], sum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = i0 + tid * per + j;
    mine[j] = j < per && i < i1 ? kept(r, l[i], i, s.tab) : 0;
    sum += mine[j];
  }
  u64 run = scan_lanes(sum);
  __syncthreads();
  if (lane == 63) s.wave[tid >> 6] = run;
  __syncthreads();
  run -= sum;
  for (int w = 0; w < tid >> 6; ++w) run += s.wave[w];
  if constexpr (kListed) {
    for (int w = 0; w < kWaves; ++w) total += s.wave[w];
    set_target();
  }
  if (target < run || target - run >= sum) return;           // one lane's range holds it
  int i = i0 + tid * per;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    run += mine[j];
    i += run <= target;
  }
  a.tokens[row] = i;
  if (a.logprobs != nullptr) a.logprobs[row] = (float)(((double)l[i] - r.top) * r.inv_t - (log((double)total) - a.bits * kLn2));
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
  if (a.V <= kSampleListed) {
    sample_pick_kernel<true><<<a.rows, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  const dim3 grid(a.n_parts, a.rows);
  sample_top_kernel<<<grid, kPartThreads, 0, stream>>>(a);
  if (a.top_k != nullptr || a.top_p != nullptr) sample_bins_kernel<<<grid, kPartThreads, 0, stream>>>(a);
  sample_parts_kernel<<<grid, kPartThreads, 0, stream>>>(a);
  sample_pick_kernel<false><<<a.rows, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace kvg
