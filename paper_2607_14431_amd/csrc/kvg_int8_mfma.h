// Device helpers of the attention kernels over int8 caches.
//
//   scores   S = (q . n_j) qstep sk: the query is an integer of 15 bits times a power of two, its upper and lower byte multiply
//            the cached integers n_j on v_mfma_i32_32x32x32_i8, exactly (|S| <= 2^14 127 256 < 2^30); a pair of these steps takes as long
//            as the one bf16 step of the same 32 dimensions would, and the cached bytes go in as they are
//   weights  w_j = p_j sv 2^x, p_j = 2^(s_j - m), rounded to fp16; x puts the row's largest weight between 2^-1 and
//            2^15, so that only weights below 2^-13 of it lose bits.  The integers m_j are exact in fp16.
#pragma once

#include "kvg_int8.h"
#include "kvg_packed_mfma.h"

#include <math.h>

namespace kvg {

namespace {

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
};
// q: the pair's query row (its first dimension), bf16; zeros for a lane without one.
template <int D>
__device__ __forceinline__ void load_query(Int8Query<D>& x, const uint16_t* q, bool ok, int half) {
  constexpr int NS = D / 32;
  uint4 raw[NS][2];
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int j = 0; j < 2; ++j) raw[s][j] = ok ? ld16(q + 32 * s + 16 * half + 8 * j) : make_uint4(0, 0, 0, 0);
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
  const int e = max(__builtin_amdgcn_frexp_expf(bf16_bits_to_f32(bits)), -100);
  const float up = finite ? __builtin_ldexpf(1.0f, 14 - e) : 0.0f;
  x.step = finite ? __builtin_ldexpf(1.0f, e - 14) : __uint_as_float(0x7FC00000u);
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

// The scales of a block of 32 keys' two pages.  A page with a scale that is not finite makes the scores NaN: value
// weights that are would reach rows that do not see it.
struct PageScales {
  float k, v, lv;              // lv: v < 2^lv
};
__device__ __forceinline__ PageScales page_scales(float k, float v) {
  const bool bad = !(fmaxf(fabsf(k), fabsf(v)) < INFINITY) || k != k || v != v;
  return {bad ? __uint_as_float(0x7FC00000u) : k, bad ? 0.0f : v, bad || v == 0.0f ? -INFINITY : (float)__builtin_amdgcn_frexp_expf(v)};
}

// Softmax state of a segment: references (log2 units, multiples of kStep) of the weights p and of p sv, and the sum of p.
struct Int8State {
  float m, mt, l;
};
// What a block does to it: factors of l and of the sums of values, the reference of its exponents, and what its pages' weights are
// multiplied with before they are rounded.
struct Int8Block {
  float alpha_l, alpha_o, m_ref, f0, f1;
  bool raised;                 // alpha_o may not be 1
};
constexpr int kWeightTop = 15;
// mx0, mx1: a row's largest scores in the block's pages, log2 units
__device__ __forceinline__ Int8Block raise_block(Int8State& s, float mx0, float mx1, const PageScales& p0, const PageScales& p1) {
  Int8Block b;
  bool up;
  b.alpha_l = raise_reference(s.m, fmaxf(mx0, mx1), up);
  b.alpha_o = raise_reference(s.mt, fmaxf(mx0 + p0.lv, mx1 + p1.lv), b.raised);
  b.m_ref = s.m == -INFINITY ? 0.0f : s.m;
  const int x = s.mt == -INFINITY ? 0 : (int)(b.m_ref - s.mt) + kWeightTop;
  // a weight of 0 times a factor past fp32's range must be 0
  b.f0 = fminf(__builtin_ldexpf(p0.v, x), 3.4e38f);
  b.f1 = fminf(__builtin_ldexpf(p1.v, x), 3.4e38f);
  return b;
}
// the power of two that takes the sums of values to the reference of the weights
__device__ __forceinline__ int end_exponent(const Int8State& s) {
  return s.mt == -INFINITY ? 0 : (int)(s.mt - s.m) - kWeightTop;
}

// A lane's 16 scores of a block from the two parts of the products, log2 units; kq: query step times the scale of page 0, 1
__device__ __forceinline__ f32x16 int8_scores(const i32x16& hi, const i32x16& lo, float kq0, float kq1) {
  f32x16 s;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (float)((hi[r] << 8) + lo[r]) * (r < 8 ? kq0 : kq1);
  return s;
}
// the largest of each page, over both halves of the wave
__device__ __forceinline__ float2 page_maxima(const f32x16& s) {
  float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int r = 0; r < 16; ++r) mx[r / 8] = fmaxf(mx[r / 8], s[r]);
  const float2 m0 = halves32(mx[0]), m1 = halves32(mx[1]);
  return make_float2(fmaxf(m0.x, m0.y), fmaxf(m1.x, m1.y));
}
// The scores' exponentials, their sum over both halves of the wave returned, and as operands of the value steps: times the pages'
// factors, rounded to fp16, each off by half a step (2^-11 of it) at most, less than the result's own rounding to bf16.
__device__ __forceinline__ float block_weights(f32x16& s, const Int8Block& b, uint4 (&p)[2]) {
  float sum[2] = {0.0f, 0.0f};
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    s[r] = __builtin_amdgcn_exp2f(s[r] - b.m_ref);
    sum[r & 1] += s[r];
  }
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const float f = w < 4 ? b.f0 : b.f1;
    (&p[w / 4].x)[w % 4] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){s[2 * w] * f, s[2 * w + 1] * f}, f16x2));
  }
  const float2 both = halves32(sum[0] + sum[1]);
  return both.x + both.y;
}

}  // namespace

}  // namespace kvg
