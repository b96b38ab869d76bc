// Device helpers of the attention kernels over int8 caches.
//
//   scores   S = (q . n_j) qstep sk: the query is an integer of 15 bits times a power of two, its upper and lower byte multiply
//            the cached integers n_j on v_mfma_i32_32x32x32_i8, exactly (|S| <= 2^14 127 256 < 2^30); a pair of these steps takes as long
//            as the one bf16 step of the same 32 dimensions would, and the cached bytes go in as they are
//   weights  w_j = p_j sv 2^x, p_j = 2^(s_j - m), rounded to fp16; x puts the row's largest weight between 2^6 and
//            2^15 (see Int8State), so that only weights below 2^-20 of it lose bits.  The integers m_j are exact in fp16.
#pragma once

#include "kvg_int8.h"
#include "kvg_packed_mfma.h"

#include <math.h>

#include <type_traits>

namespace kvg {

namespace {

// f(A), .., f(B - 1), constants: arrays that a call indexes by them stay in registers
template <int A, int B, typename F>
__device__ __forceinline__ void static_for(const F& f) {
  if constexpr (A < B) {
    f(std::integral_constant<int, A>{});
    static_for<A + 1, B>(f);
  }
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ i32x16 mfma_i8(const uint4& x, const uint4& y, const i32x16& c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, x), __builtin_bit_cast(i32x4, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma_f16(const uint4& x, const uint4& y, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

// A query as B operands of the score steps: lane (pair, half) holds dimensions 32 ss + 16 half + 0 .. 15 of step ss, value
// (256 hi + lo) step.
template <int D>
struct Int8Query {
  uint4 hi[D / 32], lo[D / 32];
  float step;
  bool finite;
};
// q: the pair's query row (its first dimension), bf16; a lane without a pair takes another's.
template <int D>
__device__ __forceinline__ void load_query(uint4 (&raw)[D / 32][2], const uint16_t* q, int half) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s)
#pragma unroll
    for (int j = 0; j < 2; ++j) raw[s][j] = ld16(q + 32 * s + 16 * half + 8 * j);
}
template <int D>
__device__ __forceinline__ void split_query(Int8Query<D>& x, const uint4 (&raw)[D / 32][2]) {
  constexpr int NS = D / 32;
  u16x2 most = {0, 0};
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int w = 0; w < 8; ++w)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, (&raw[s][w / 4].x)[w % 4] & 0x7FFF7FFFu));
  const uint32_t mine = most.x > most.y ? most.x : most.y;
  const auto both = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
  const uint32_t bits = both[0] > both[1] ? both[0] : both[1];         // of the largest |q|; Inf and NaN above all others
  const bool finite = bits < 0x7F80u;
  // |q| < 2^e; below 2^-100 the integers get smaller
  const int e = finite ? max(__builtin_amdgcn_frexp_expf(bf16_bits_to_f32(bits)), -100) : 0;
  const float up = finite ? __builtin_ldexpf(1.0f, 14 - e) : 0.0f;
  x.step = __builtin_ldexpf(1.0f, e - 14);
  x.finite = finite;
  // q up + 1.5 2^23 has the integer, rounded to nearest even, in its low bits; 128 more and its byte 1 is the upper byte that
  // goes with a signed lower one
  constexpr float kRound = 12582912.0f;
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int w = 0; w < 4; ++w) {                                      // four dimensions: words 2 w and 2 w + 1 of the raw ones
      uint32_t lo[2], hi[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t r = finite ? (&raw[s][w / 2].x)[2 * (w % 2) + j] : 0u;
        const float a = fmaf(__uint_as_float(r << 16), up, kRound), b = fmaf(__uint_as_float(r & 0xFFFF0000u), up, kRound);
        lo[j] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0C0C0400u);
        hi[j] = __builtin_amdgcn_perm(__float_as_uint(b + 128.0f), __float_as_uint(a + 128.0f), 0x0C0C0501u);
      }
      (&x.lo[s].x)[w] = lo[0] | lo[1] << 16;
      (&x.hi[s].x)[w] = hi[0] | hi[1] << 16;
    }
}

// K fragment of step ss (32 rows x 32 dims, 16 a lane) at the lane's base, k_lane_base<D, false>.
template <int D>
__device__ __forceinline__ uint4 int8_k_fragment(const lds_char* lane_base, int ss) {
  return k_fragment<D, false>(lane_base, ss);
}

// eight integers -> fp16, exactly: 0x6400 | (n + 128) is 1024 + n + 128
__device__ __forceinline__ uint4 widen_int8(const uint2& x) {
  uint4 r;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t w = (j ? x.y : x.x) ^ 0x80808080u;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, k ? 0x04030402u : 0x04010400u));
      (&r.x)[2 * j + k] = __builtin_bit_cast(uint32_t, h - (f16x2){(_Float16)1152.0f, (_Float16)1152.0f});
    }
  }
  return r;
}

// A page's scales as the kernels use them, a page a lane; ones that are not finite count as 0 (`bad`: rows that see a token of
// the page get NaN).
struct PageScales {
  float k, lv;                 // lv: log2 of the values' scale, -Inf for a block of zeros
  bool bad;
};
__device__ __forceinline__ PageScales page_scales(float k, float v) {
  const bool bad = !(fabsf(k) < INFINITY) || !(fabsf(v) < INFINITY);
  return {bad ? 0.0f : k, bad ? -INFINITY : __builtin_amdgcn_logf(v), bad};
}
__device__ __forceinline__ float lane_value(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

constexpr float kNaN = __builtin_nanf("");

// Softmax state of a segment: the reference m of the weights p = 2^(s - m) (log2 units, a multiple of kStep), the sum of p (l0 at first: 0,
// or NaN for a query that is not finite), m_ref: m, or 0 before the first key, the exponent x that takes p sv to the range of fp16, and
// mt, what s + log2 sv has to pass for another x (-Inf: no value yet).  The reference of p sv is the integer r = kWeightTop - x.
//
// Weights are p sv 2^x = 2^(S kq + c), all below 2^kWeightTop and rounded to fp16: off by half a step (2^-11 of it) at
// most, less than the result's own rounding to bf16.  r goes kRoom above what raises it, so that later blocks seldom raise it again (all
// of a wave's sums are multiplied where one of its rows does; with 4 in place of 8, 7% more vector instructions): the largest weight is above 2^6, and
// those below 2^-20 of it lose bits.  p is the weight times `back`.  Values that weigh less than 2^-kLightest of the row's largest
// may as well weigh that: it stays far below an fp16 step, and the sum of p keeps its bits.
constexpr float kWeightTop = 15.0f, kRoom = 8.0f, kLightest = 60.0f;
// Rows whose m is past this are far out: see far_page.
constexpr float kFar = 0x1p20f;
struct Int8State {
  float m, mt, l, m_ref, x;
};
__device__ __forceinline__ Int8State empty_state(float l0) { return {-INFINITY, -INFINITY, l0, 0.0f, 0.0f}; }
__device__ __forceinline__ bool is_far(const Int8State& st) { return fabsf(st.m_ref) >= kFar; }

// The larger of both halves of the wave, of x and of y.
__device__ __forceinline__ float2 max_halves(float x, float y) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);      // lower halves, upper ones
  const float m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));                                       // of x below, of y above
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return make_float2(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The steps of a block of 32 keys (two pages).  A lane's scores of a page are S kq: S an integer (as a float; -Inf for a key that
// the row does not see), kq the query's step times the keys' scale, in log2 units (not 0, by which -Inf would be NaN, and not above
// 2^96, by which |S| < 2^30 would leave fp32).
__device__ __forceinline__ float key_factor(float q_scale, float k) { return __builtin_amdgcn_fmed3f(q_scale * k, 0x1p-126f, 0x1p96f); }
// A lane's largest score of a page, rounded to fp32: what the references are raised by, in every kernel.
__device__ __forceinline__ float largest_score(float S, float kq) {
#pragma clang fp contract(off)
  return S * kq;
}
// Whether a lane's largest scores of the pages (both halves of the wave joined) raise its references.  The one test of that: a wave
// takes its rows to raise_block() together, but the rows whose own test fails keep their state, so that a row's bytes are
// those it has alone.  (No fma here: sums of rounded products are the same in every kernel.)
__device__ __forceinline__ bool is_raised(const Int8State& s, float mx0, float mx1, float lv0, float lv1) {
#pragma clang fp contract(off)
  return fmaxf(mx0, mx1) > s.m || fmaxf(mx0 + lv0, mx1 + lv1) > s.mt;
}
// What they do to the state where `raised` (is_raised): factors of the sum of p and of the sums of values, powers of two (or 0), and
// 1 elsewhere.  mx + lv rounds by up to 2^-4 (below kFar), so weights of a row that is not raised stay below 2^(kWeightTop + 1/16).
struct Int8Raise {
  float alpha_l, alpha_o;
};
__device__ __forceinline__ Int8Raise raise_block(Int8State& s, bool raised, float mx0, float mx1, float lv0, float lv1) {
#pragma clang fp contract(off)
  Int8State to = s;
  Int8Raise b;
  bool up;
  b.alpha_l = raise_reference(to.m, fmaxf(mx0, mx1), up);
  to.m_ref = to.m == -INFINITY ? 0.0f : to.m;
  const float was = s.mt == -INFINITY ? -INFINITY : kWeightTop - s.x + (s.m - to.m);      // r beside the new m
  const float y = fmaxf((mx0 - to.m_ref) + lv0, (mx1 - to.m_ref) + lv1), at = __builtin_ceilf(y) + kRoom;
  up = y > was;
  b.alpha_o = up ? __builtin_amdgcn_exp2f(was - at) : 1.0f;
  const float r = up ? at : was;
  to.x = r == -INFINITY ? 0.0f : kWeightTop - r;
  // far out, the sum s + log2 sv has no bits to compare: every block comes here
  to.mt = r == -INFINITY ? r : is_far(to) ? -0x1p127f : r + to.m_ref;
  s.m = raised ? to.m : s.m;
  s.mt = raised ? to.mt : s.mt;
  s.m_ref = raised ? to.m_ref : s.m_ref;
  s.x = raised ? to.x : s.x;
  return {raised ? b.alpha_l : 1.0f, raised ? b.alpha_o : 1.0f};
}
struct Int8Page {
  float c, back;
};
__device__ __forceinline__ Int8Page page_weights(const Int8State& s, float lv) {
  const float f = fmaxf(lv + s.x, -kLightest);
  return {f - s.m_ref, __builtin_amdgcn_exp2f(-f)};
}
// Rows whose reference is so far out that a score's rounding is past a few units: the exact product S kq of fma could lie well above or
// below the rounded one that the reference was raised to, and every weight be Inf or 0.  Their scores are rounded, and taken less the
// reference, which is exact near it; `first`: of a page's eight in s.  (the other rows keep theirs)
__device__ __forceinline__ void far_page(f32x16& s, int first, float& kq, Int8Page& p, const Int8State& st, float lv) {
#pragma clang fp contract(off)
  const bool far = is_far(st);
#pragma unroll
  for (int r = first; r < first + 8; ++r) {
    const float rounded = s[r] * kq;
    s[r] = far ? rounded - st.m_ref : s[r];
  }
  kq = far ? 1.0f : kq;
  p.c = far ? fmaxf(lv + st.x, -kLightest) : p.c;
}
__device__ __forceinline__ float weight_of(float S, float kq, float c) { return __builtin_amdgcn_exp2f(fmaf(S, kq, c)); }
__device__ __forceinline__ uint32_t round_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
}
// eight weights as an operand of the value steps
__device__ __forceinline__ uint4 round_weights8(const f32x16& s, int h) {
  return make_uint4(round_pair(s[8 * h], s[8 * h + 1]), round_pair(s[8 * h + 2], s[8 * h + 3]), round_pair(s[8 * h + 4], s[8 * h + 5]),
                    round_pair(s[8 * h + 6], s[8 * h + 7]));
}
// The block's part of the sum of p from a lane's sums of weights of the pages (both halves of the wave).
__device__ __forceinline__ float block_sum(float sum0, float sum1, float back0, float back1) {
  const float2 both = halves32(fmaf(sum0, back0, sum1 * back1));
  return both.x + both.y;
}
// End of a segment: the exponent that takes its sums of values to p sv (far below fp32 where every scale was 0).
__device__ __forceinline__ int end_exponent(const Int8State& s) { return s.mt == -INFINITY ? -1000 : (int)fmaxf(-s.x, -1000.0f); }

}  // namespace

}  // namespace kvg
