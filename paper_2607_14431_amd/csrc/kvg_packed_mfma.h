// Device helpers of the packed sequences' MFMA attention kernels: references, LDS layout, values that are not finite,
// the fold of segment states.
#pragma once

#include "kvg_mfma.h"
#include "kvg_packed.h"
#include "kvg_rows.h"

#include <math.h>

namespace kvg {

namespace {

constexpr float kStep = 8.0f;          // grid of the references, log2 units

// The reference that a largest score (log2 units) asks for.
__device__ __forceinline__ float reference_of(float mx) { return ceilf(mx * (1.0f / kStep)) * kStep; }

// LDS rows hold their 16-byte chunks at position chunk ^ swizzle(row), XOR-linear in the row bits.  K is read as one chunk
// of 32 consecutive rows per lane half, V transposed (bf16: four rows x two or four chunks, fp8: rows
// {0..3, 8..11} (+ 4) of a 16-row step).
template <int RB, bool kFp8>
struct SwzTile {
  __device__ static __forceinline__ int k(int r) {
    if constexpr (kFp8) return RB == 256 ? (r & 15) : RB == 128 ? ((r >> 1) & 7) : ((r >> 2) & 3);
    return RB >= 256 ? (r & 15) : (r & 7);
  }
  __device__ static __forceinline__ int v(int r) {
    if constexpr (kFp8)
      return RB == 256 ? (r & 15) : RB == 128 ? (((r >> 1) & 1) | (((r >> 3) & 1) << 1)) : ((r >> 3) & 1);
    return RB >= 256 ? ((0xCA60 >> (4 * (r & 3))) & 15) : 2 * (r & 3);
  }
};

__device__ __forceinline__ float load_value(const uint16_t* p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ float load_value(const uint8_t* p) { return Elem<uint8_t>::get(make_uint4(*p, 0, 0, 0), 0); }

// whether one of the values is Inf or NaN (bf16: all exponent bits set)
__device__ __forceinline__ bool bad_values(const uint4& x, uint16_t) {
  bool bad = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t v = (&x.x)[w];
    bad = bad || (v & 0x7F80u) == 0x7F80u || (v & 0x7F800000u) == 0x7F800000u;
  }
  return bad;
}
// fp8: NaN codes 0x7F and 0xFF
__device__ __forceinline__ bool bad_values(const uint4& x, uint8_t) {
  uint32_t m = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) m |= ((&x.x)[w] & 0x7F7F7F7Fu) + 0x01010101u;
  return (m & 0x80808080u) != 0;
}

// The page of value rows at p with every Inf and NaN set to 0; whether there was one.
template <typename T, int NCH>
__device__ __forceinline__ bool finite_rows(uint4* p, int lane) {
  bool any = false;
#pragma unroll 2
  for (int i = lane; i < kPage * NCH; i += 64) {
    uint4 x = p[i];
    if (!bad_values(x, T{})) continue;
    any = true;
    T* v = reinterpret_cast<T*>(p + i);
    for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
      if (!(fabsf(load_value(v + e)) < INFINITY)) v[e] = 0;
  }
  return __builtin_amdgcn_ballot_w64(any) != 0;
}

__device__ __forceinline__ f32x16 splat(float x) { return (f32x16)(x); }

__device__ __forceinline__ f32x16 mfma32(const uint4& x, const uint4& y, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x), as_bf16x8(y), c, 0, 0, 0);
}

// K fragment ss of 32 rows whose lane base is `lane`: eight values of head_dim for each lane's row (fp8 widened).
template <bool kFp8>
__device__ __forceinline__ uint4 k_fragment(const lds_char* rows, uint32_t lane, int ss) {
  if constexpr (kFp8) {
    const u32x2 w = *reinterpret_cast<const lds_u32x2*>(rows + (lane ^ (uint32_t)(16 * ss)));
    return widen_fp8x8(w.x, w.y);
  } else {
    return __builtin_bit_cast(uint4, *reinterpret_cast<const lds_u32x4*>(rows + (lane ^ (uint32_t)(32 * ss))));
  }
}
// V^T fragment of 16 rows, dims 32 d .. 32 d + 31.
template <int RB, bool kFp8>
__device__ __forceinline__ uint4 v_fragment(const lds_char* rows, uint32_t lane, int d) {
  if constexpr (kFp8) {
    const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(rows + (lane ^ (uint32_t)(32 * d))));
    return widen_fp8x8((uint32_t)w.x, (uint32_t)w.y);
  } else {
    const uint32_t at = lane ^ (uint32_t)(64 * d);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(rows + at));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(rows + at + 8 * RB));
    const uint2 lo2 = __builtin_bit_cast(uint2, lo), hi2 = __builtin_bit_cast(uint2, hi);
    return make_uint4(lo2.x, lo2.y, hi2.x, hi2.y);
  }
}
// The lane's base in 32 K rows, and in 16 V rows:
//   K  row lane % 32, chunk 2 ss + lane / 32 (fp8: 8 bytes at 16 ss + 8 (lane / 32))
//   V  16-lane group tr_m = lane / 16, tr_k = lane % 16: bf16 rows 4 (tr_m / 2) + tr_k / 4 (and 8 further), 8 bytes at dim
//      32 d + 16 (tr_m % 2) + 4 (tr_k % 4); fp8 row 4 (tr_m / 2) + {0..3, 8..11}[tr_k / 2], 8 bytes at dim
//      32 d + 16 (tr_m % 2) + 8 (tr_k % 2)
template <int RB, bool kFp8>
__device__ __forceinline__ uint32_t k_lane_base(int lane) {
  using SW = SwzTile<RB, kFp8>;
  const int r = lane & 31, half = lane >> 5;
  return kFp8 ? r * RB + 16 * SW::k(r) + 8 * half : r * RB + 16 * (half ^ SW::k(r));
}
template <int RB, bool kFp8>
__device__ __forceinline__ uint32_t v_lane_base(int lane) {
  using SW = SwzTile<RB, kFp8>;
  const int tr_k = lane & 15, tr_m = lane >> 4;
  if constexpr (kFp8) {
    const int kk = 4 * (tr_m >> 1) + ((tr_k >> 1) & 3) + 8 * (tr_k >> 3);
    return kk * RB + 16 * ((tr_m & 1) ^ SW::v(kk)) + 8 * (tr_k & 1);
  } else {
    const int rr = (tr_m >> 1) * 4 + (tr_k >> 2);
    return rr * RB + 8 * (tr_k & 1) + 16 * ((2 * (tr_m & 1) + ((tr_k & 3) >> 1)) ^ SW::v(rr));
  }
}

// Softmax state of a segment's blocks of 32 keys; the operations of one block, in the order every kernel takes them.
// The reference after a block whose largest score (log2 units) is mx; returns what the sums so far are
// multiplied with, exactly 1 where the reference stays.
__device__ __forceinline__ float raise_reference(float& m, float mx, bool& raised) {
  raised = mx > m;
  const float up = reference_of(mx);
  const float alpha = raised ? __builtin_amdgcn_exp2f(m - up) : 1.0f;
  m = raised ? up : m;
  return alpha;
}
// eight weights (a lane's scores of a block, elements 8 h ..) as a bf16 operand, their sum added to psum as rounded
__device__ __forceinline__ uint4 round_weights(const f32x16& p, int h, float& psum) {
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  uint4 f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    (&f.x)[w] = pack_bf16_rne(p[8 * h + 2 * w], p[8 * h + 2 * w + 1]);
    psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (&f.x)[w]), ones, psum, false);
  }
  return f;
}
// Rows of the few kernel's sequences before sequence b (a wave's lanes together).
__device__ __forceinline__ int few_rows_before(const PackedAttnArgs& a, int b) {
  int rows = 0;
  for (int i = __lane_id(); i < b; i += 64) {
    const SeqRange r = seq_range(a.seqs, i);
    rows += is_few(a, r) ? r.len : 0;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) rows += __shfl_xor(rows, d);
  return __builtin_amdgcn_readfirstlane(rows);
}

// a state folded into the running one (reference, sum): what both are multiplied with
struct FoldFactors {
  float run, part;
};
__device__ __forceinline__ FoldFactors fold_factors(float& m_run, float& l_run, float m, float l) {
  const float m_new = fmaxf(m_run, m);
  const FoldFactors f = {merge_factor(m_run, m_new), merge_factor(m, m_new)};
  m_run = m_new;
  l_run = fmaf(l, f.part, l_run * f.run);
  return f;
}

}  // namespace

}  // namespace kvg
