// Tokens from logits: temperature, top-k, top-p, min-p and given random numbers.
//
// With x_i = (l_i - max l) / T in fp64 a token weighs e^x_i, rounded to fixed point with `bits` bits after the point: sums of a
// row's weights are integers below 2^62, so they have no order and no rounding.  Tokens are ordered by a
// code of 56 bits, the logit's (32 bits that compare as the floats do) over the inverted index: the likelier first, of equal
// ones the lower index.  Each limit keeps a prefix of that order: top-k ends at the k-th largest code, top-p where the running sum
// of weights reaches its share, min-p at a weight.  So what is kept is `code >= cut && e^x >= min_p`, and the token is the first in
// index order whose running sum of kept weights passes the random number's.
//
// Rows of up to kSampleListed tokens: a workgroup holds the row's codes (4,096 tokens, us, without limits / top-k / top-p / both: one row 8 / 11 / 17 /
// 19, 256 rows 8 / 12 / 30 / 32: the chain of select()'s passes, each a round over LDS with five barriers).  Longer ones in passes over the row, by
// many workgroups:
//   top     the largest logit of every part of the row
//   bins    count and weight of the row's tokens by weight (1,024 equal steps of the exponent down to weight 0), where a top-k or
//           top-p may end inside the row.  The bins tell in which of them the two limits end.  Weights are left out where top-p is 1
//           or the tokens of top-k are few (by_list): an exponential in fp64 costs more than all else in the pass
//   parts   the weight of every part's tokens in the bins before those, and a list of the codes in them
//   pick    a workgroup a row: the list gives the cut; the parts' weights the part that holds the token, which is searched
// Bound: one row, four launches and the chains in them (262,144 tokens: 3 + 8 + 5 + 10 us; a workgroup that makes every pass took
// 523).  64 rows, each with other limits: 13 us for the first read (5.2 TB/s), 22 for the bins (fp64 exponentials and LDS
// additions of the rows with a top-p alone), 18 for the parts, 24 for the longest lists.  A bitonic sort of a list of 1,400 codes
// took 20 us, select() about 5.
//
// Where the list would be too long the cut is found digit by digit instead (11, 11, 10 bits of the logit, twice 12 of the index): count or
// weight of the tokens that share the digits so far, by their next digit.  One workgroup makes these passes over the row, five for each
// limit.  That takes more than 4,096 tokens in the bins where the limits end, (bits + 2) ln 2 / 1,024 wide in x each (0.031 at 262,144
// tokens): equal logits, but flat rows too, normal ones of sigma / T below about 0.65 with a top-p of 0.9, wider ones of longer
// vocabularies.  262,144 tokens with that top-p, us, at sigma / T of 3 / 0.75 / 0.5 / equal logits: one row 33 / 37 / 641 / 1,289, 64 rows 103 / 109 /
// 925 / 2,687; 32,000 tokens, 3 / 0.3 / equal: one row 24 / 29 / 198, 64 rows 39 / 45 / 348; one row of 2,097,152, 3 / 0.5: 64 / 6,489.
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
constexpr int kFew = 128;                 // codes that a wave sorts, two a lane
struct Shared {
  double tab[64];
  u64 wave[kWaves];
  u64 found[2];
  union {
    Digits digits;
    struct {
      u64 hi[kWaves], lo[kWaves], bins[kThreads], found, before;
      uint32_t n;
    } select;
  };
  u64 few[2 * kFew];                  // unsorted, sorted
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
  r.least = fmaxf(r.least - fabsf(r.least) * 0x1p-22f - 1e-37f, -3.4028235e38f);
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
  u64 weight[16];             // of the waves' bins
  uint32_t count[16];
  u64 upto_k;                 // weight up to top-k's bin, with it
  Ends ends;
};
// A lane's bins, in order; requested before what the row's parameters wait for.
template <int kT>
struct LaneBins {
  static constexpr int kPer = kSampleBins / kT;
  u64 w[kPer];
  uint32_t c[kPer];
  __device__ __forceinline__ void load(const SampleArgs& a, int row) {
    const int64_t at = (int64_t)row * kSampleBins + threadIdx.x * kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      w[i] = a.bin_weights[at + i];
      c[i] = a.bin_counts[at + i];
    }
  }
};
// (all lanes of a workgroup of kSampleBins lanes or fewer)
template <int kT>
__device__ void find_ends(const SampleArgs& a, int row, const LaneBins<kT>& bins, Ends& out, EndsShared& s) {
  constexpr int kPer = kSampleBins / kT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = threadIdx.x * kPer;
  const u64(&w)[kPer] = bins.w;
  const uint32_t(&c)[kPer] = bins.c;
  u64 sw = 0;
  uint32_t sc = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    sw += w[i];
    sc += c[i];
  }
  u64 uw = sw;                                               // up to and with this lane's
  uint32_t uc = sc;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const u64 x = __shfl_up(uw, m);
    const uint32_t y = __shfl_up(uc, m);
    uw += lane >= m ? x : 0;
    uc += lane >= m ? y : 0;
  }
  if (lane == 63) {
    s.weight[wave] = uw;
    s.count[wave] = uc;
  }
  if (threadIdx.x == 0) s.ends = {0, -1, kSampleBins, 0, 0, 0, 0};
  __syncthreads();
  u64 total_w = 0;
  uint32_t total_c = 0;
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
  const bool by_k = k > 0 && (uint32_t)k < total_c;
  if (by_k) {
    u64 x = uw;
    uint32_t y = uc;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (y < (uint32_t)k && y + c[i] >= (uint32_t)k) {
        s.ends.k_bin = b0 + i;
        s.ends.k_need = (uint32_t)k - y;
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
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) n += b0 + i >= s.ends.first && b0 + i <= s.ends.last && b0 + i < s.ends.k_bin ? c[i] : 0;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) n += __shfl_xor(n, m);
    if (lane == 0 && n != 0) atomicAdd(&s.ends.listed_before_k, n);
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
  LaneBins<kPartThreads> bins;
  bins.load(a, row);
  Row r;
  if (!row_setup(a, row, row_top(a, row), false, r)) return;
  if (threadIdx.x < 64) tab[threadIdx.x] = exp2(threadIdx.x / 64.0);
  Ends ends = {kSampleBins, -1, kSampleBins, 0, 0, 0, 0};
  if (limited(a, row)) find_ends<kPartThreads>(a, row, bins, ends, ends_shared);
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

// Up to and with each lane's, in order.
__device__ __forceinline__ u64 scan_lanes(u64 x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const u64 before = __shfl_up(x, m);
    x += (int)(threadIdx.x & 63) >= m ? before : 0;
  }
  return x;
}

__device__ __forceinline__ u64 code_weight(const Row& r, u64 c, const double* tab) {
  return weight(r, logit_of((uint32_t)(c >> kSampleIndexBits)), tab).n;
}
// Up to kFew codes in the first wave, without a barrier: the largest first, lane i has the ones at 2 i and 2 i + 1 (0: none).
struct Few {
  u64 a, b;
  __device__ __forceinline__ u64 at(int i) const { return __shfl(i & 1 ? b : a, i >> 1); }
};
__device__ __forceinline__ u64 from_lane(u64 x, int j) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, j), hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), j);
  return (u64)hi << 32 | lo;
}
// a, b: the lane's, the codes at `lane` and `lane + 64` of n (the wave's)
__device__ __forceinline__ Few sort_few(u64 a, u64 b, int n, u64* sorted) {
  const int lane = threadIdx.x & 63;
  int at_a = 0, at_b = 0;
  for (int j = 0; j < min(n, 64); ++j) {
    const u64 c = from_lane(a, j);
    at_a += c > a;
    at_b += c > b;
  }
  for (int j = 0; j < n - 64; ++j) {
    const u64 c = from_lane(b, j);
    at_a += c > a;
    at_b += c > b;
  }
  if (lane < n) sorted[at_a] = a;
  if (lane + 64 < n) sorted[at_b] = b;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return {2 * lane < n ? sorted[2 * lane] : 0, 2 * lane + 1 < n ? sorted[2 * lane + 1] : 0};
}
// The first place at which the weights wa, wb up to it reach `need`; n - 1 if none.
__device__ __forceinline__ int reach_few(u64 wa, u64 wb, u64 need, int n) {
  const u64 upto = scan_lanes(wa + wb);
  const uint64_t past = __builtin_amdgcn_ballot_w64(upto >= need);
  if (past == 0) return n - 1;
  const int at = __builtin_ctzll(past);
  return min(2 * at + (__shfl(upto - wb, at) < need), n - 1);
}

// The sum over the workgroup.  (all lanes)
__device__ u64 sum_block(u64 x, Shared& s) {
  x = add_lanes(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = x;
  __syncthreads();
  u64 total = 0;
  for (int w = 0; w < kWaves; ++w) total += s.wave[w];
  return total;
}

// Listed codes of a lane (0: none).
constexpr int kHeld = kSampleListed / kThreads;
// The code at which the count (or, by_weight, the weight) of the codes, from the largest on, reaches `need`; the least one if it does not.
// The codes are put into bins by their logit, linearly between `high` and `low`, and all but those of the bin where that happens are
// dropped; so on between the largest and the least of the rest, by index where their logits are equal, until kFew are left.  (all
// lanes; finite logits, of which none need lie at or between the ends; the next call may follow at once)
__device__ u64 select(const Row& r, const u64 (&codes)[kHeld], bool by_weight, u64 need, double high, double low, Shared& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto& t = s.select;
  u64 c[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) c[j] = codes[j];
  bool equal = false;
  double first = high, range = high - low;
  while (true) {
    __syncthreads();
    t.bins[tid] = 0;
    if (tid == 0) t.n = 0;
    __syncthreads();
    auto value = [&](u64 x) -> double { return equal ? (double)(x & kIndexMask) : (double)logit_of((uint32_t)(x >> kSampleIndexBits)); };
    const double scale = range > 0.0 ? (kThreads - 1) / range : 0.0;
    auto bin = [&](u64 x) -> int { return (int)fmin(fmax((first - value(x)) * scale, 0.0), (double)(kThreads - 1)); };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (c[j] != 0) atomicAdd(&t.bins[bin(c[j])], by_weight ? code_weight(r, c[j], s.tab) : 1);
    __syncthreads();
    const u64 mine = t.bins[tid];
    u64 upto = scan_lanes(mine);
    if (lane == 63) s.wave[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += s.wave[w];
    if (upto - mine < need && (upto >= need || tid == kThreads - 1)) {
      t.found = (u64)tid;
      t.before = upto - mine;
    }
    __syncthreads();
    need -= t.before;
    const int found = (int)t.found;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (c[j] != 0) {
        if (bin(c[j]) != found) {
          c[j] = 0;
        } else {
          const uint32_t at = atomicAdd(&t.n, 1u);
          if (at < kFew) s.few[at] = c[j];
        }
      }
    __syncthreads();
    if (t.n <= kFew) break;
    u64 most = 0, least = 0;                                 // least: of the inverted codes
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      most = c[j] > most ? c[j] : most;
      least = c[j] != 0 && ~c[j] > least ? ~c[j] : least;
    }
    most = max_lanes(most);
    least = max_lanes(least);
    if (lane == 0) {
      t.hi[wave] = most;
      t.lo[wave] = least;
    }
    __syncthreads();
    most = max_lanes(lane < kWaves ? t.hi[lane] : 0);
    least = ~max_lanes(lane < kWaves ? t.lo[lane] : 0);
    equal = most >> kSampleIndexBits == least >> kSampleIndexBits;
    first = equal ? (double)(most & kIndexMask) : (double)logit_of((uint32_t)(most >> kSampleIndexBits));
    range = first - (equal ? (double)(least & kIndexMask) : (double)logit_of((uint32_t)(least >> kSampleIndexBits)));
  }
  if (tid < 64) {
    const int n = __builtin_amdgcn_readfirstlane((int)t.n);
    const Few x = sort_few(lane < n ? s.few[lane] : 0, lane + 64 < n ? s.few[lane + 64] : 0, n, s.few + kFew);
    const int at = by_weight ? reach_few(2 * lane < n ? code_weight(r, x.a, s.tab) : 0, 2 * lane + 1 < n ? code_weight(r, x.b, s.tab) : 0, need, n)
                             : (int)min(need, (u64)n) - 1;
    t.found = x.at(at);
  }
  __syncthreads();
  return t.found;
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
  u64 top = 0, early[2] = {0, 0};                            // early: the first listed codes
  uint32_t n_listed = 0;
  LaneBins<kThreads> bins;
  if constexpr (kListed) {
    for (int i = tid; i < a.V; i += kThreads) {
      const u64 c = token_code(l[i], i);
      top = c > top ? c : top;
    }
    top = max_lanes(top);
    if (lane == 0) s.wave[tid >> 6] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = s.wave[w] > top ? s.wave[w] : top;
    __syncthreads();
  } else {
    bins.load(a, row);
    n_listed = __builtin_amdgcn_readfirstlane((int)a.n_listed[row]);
    early[0] = a.listed[(int64_t)row * kSampleListed + lane];
    early[1] = a.listed[(int64_t)row * kSampleListed + 64 + lane];
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
      u64 c[kHeld], sum = 0;
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int i = tid + j * kThreads;
        c[j] = i < a.V && l[i] >= r.least ? token_code(l[i], i) : 0;
      }
      if (k > 0 && k < a.V) r.cut = select(r, c, false, (u64)k, r.top, r.least, s);
      if (p < 1.0f) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) sum += c[j] != 0 && c[j] >= r.cut ? code_weight(r, c[j], s.tab) : 0;
        r.cut = select(r, c, true, share_of(p, sum_block(sum, s)), r.top, r.least, s);
      }
    }
  } else {
    Ends ends = {kSampleBins, -1, kSampleBins, 0, 0, 0, 0};
    if (limit) find_ends<kThreads>(a, row, bins, ends, ends_shared);
    searched = !limit || n_listed <= kSampleListed;
    if (!searched) {
      if (k > 0 && k < a.V) r.cut = find_cut(a, r, l, false, (u64)k, s);
      if (p < 1.0f) {
        Row whole = r;
        whole.min_p = 0.0;
        r.cut = find_cut(a, r, l, true, share_of(p, part_weights(whole, l, 0, a.V, (a.V + kWaves - 1) / kWaves, s)), s);
      }
    } else if (ends.first < kSampleBins) {
      // n: listed tokens of top-k.  What top-p has a share of: `base` and, where top-k or by_list say, the weight of those of them that
      // no bin's weight holds
      const bool by_k = ends.k_bin < kSampleBins, whole = by_list(a, row), add = by_k || whole;
      int n = by_k ? (int)(ends.listed_before_k + ends.k_need) : (int)n_listed;
      u64 base = by_k ? ends.before_k : 0;
      if (!add)
        for (int i = 0; i < kWaves; ++i) base += ends_shared.weight[i];
      auto to_part = [&](u64 c) {                            // a listed token that is kept, to its part
        const Weight w = weight(r, logit_of((uint32_t)(c >> kSampleIndexBits)), s.tab);
        if (w.e >= r.min_p) atomicAdd(&parts[token_of(c) / a.part_size], w.n);
      };
      if (n_listed <= kFew && tid >= 64) {
      } else if (n_listed <= kFew) {
        const int all = (int)n_listed, i = 2 * lane;
        const Few x = sort_few(lane < all ? early[0] : 0, lane + 64 < all ? early[1] : 0, all, s.few);
        if (p < 1.0f) {
          u64 wa = i < n ? code_weight(r, x.a, s.tab) : 0, wb = i + 1 < n ? code_weight(r, x.b, s.tab) : 0;
          const int from = by_k && !whole ? (int)ends.listed_before_k : 0;
          if (add) base += add_lanes((i >= from ? wa : 0) + (i + 1 >= from ? wb : 0));
          n = reach_few(wa, wb, share_of(p, base) - ends.before_first, n) + 1;
        }
        r.cut = x.at(n - 1);
        if (i < n) to_part(x.a);
        if (i + 1 < n) to_part(x.b);
        s.found[0] = r.cut;
      } else {
        u64 c[kHeld], sum = 0;
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
          const int i = tid + j * kThreads;
          c[j] = i < (int)n_listed ? a.listed[(int64_t)row * kSampleListed + i] : 0;
        }
        const double bin = 1.0 / (r.inv_t * r.bin_scale), high = r.top - ends.first * bin;
        const double low = r.top - (max(ends.last, by_k ? ends.k_bin : 0) + 1) * bin;
        if (by_k) r.cut = select(r, c, false, (u64)n, high, low, s);
        if (p < 1.0f) {
          if (add) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
              if (c[j] != 0 && c[j] >= r.cut && (whole || bin_of(r, logit_of((uint32_t)(c[j] >> kSampleIndexBits))) == ends.k_bin))
                sum += code_weight(r, c[j], s.tab);
            base += sum_block(sum, s);
          }
          r.cut = select(r, c, true, share_of(p, base) - ends.before_first, high, low, s);
        }
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
          if (c[j] != 0 && c[j] >= r.cut) to_part(c[j]);
      }
    }
    __syncthreads();
    if (limit && n_listed <= kFew && ends.first < kSampleBins) r.cut = s.found[0];
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
