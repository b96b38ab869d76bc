// Device helpers of the kernels that rotate packed rows: angles, places of a head's values in the rotation, sums over the
// lanes of a head.
#pragma once

#include "kvg_mfma.h"
#include "kvg_packed.h"

#include <type_traits>

namespace kvg {

namespace {

// Results are written past the caches (those prompts 102.5 us, 106.5 with plain stores; the block rotated 16.5, 19.6), raw rows are
// read through them, where a projection may just have written them (nontemporal: the prompts 101.7, the block 19.2).
__device__ __forceinline__ void st16s(void* p, const uint4& v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ uint4 ld16(const void* p) { return *reinterpret_cast<const uint4*>(p); }

// (cos, sin) of pos * theta_i times the amplitude
__device__ __forceinline__ float2 turn(const RotaryArgs& r, int64_t pos, int i) {
  double s, c;
  sincos((double)pos * r.theta[i], &s, &c);
  return make_float2((float)(c * r.amplitude), (float)(s * r.amplitude));
}

// The position pair i of packed row `row` turns by: the token's own (`pos`), or that of the pair's axis.
template <typename Axes>
__device__ __forceinline__ int64_t pair_position(const Axes& axes, int64_t pos, int64_t row, int64_t n_rows, int i) {
  if constexpr (std::is_same<Axes, AxesArgs>::value)
    return axes.positions[axes.axis[i] * n_rows + row];
  else
    return pos;
}

// Where the values e0 .. e0 + E - 1 of a head go in the rotation: the offset of the vector that holds their
// partners (their own for interleaved pairs and for values that are not rotated).
struct Place {
  bool rotated, first;
  int partner, pair;          // pair: index of the first value's pair
};
__device__ __forceinline__ Place place(const RotaryArgs& r, int e0) {
  const int half = r.dim >> 1;
  Place p;
  p.rotated = e0 < r.dim;
  p.first = r.pairing != 0 || e0 < half;
  p.partner = !p.rotated || r.pairing != 0 ? e0 : p.first ? e0 + half : e0 - half;
  p.pair = r.pairing != 0 ? e0 >> 1 : p.first ? e0 : p.partner;
  return p;
}

// y: the values of this lane's partners (half pairing), from the lane of the head that holds them in x
template <int E>
__device__ __forceinline__ void from_partner(const Place& p, int e0, const float (&x)[E], float (&y)[E]) {
  const int from = 4 * ((int)(threadIdx.x & 63) + (p.partner - e0) / E);
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)__float_as_uint(x[e])));
}

// x: the vector's values, y: its partners' (half pairing); the operations of rotate_pair()
template <int E>
__device__ __forceinline__ void rotate_values(const Place& p, int pairing, const float2* cs, float (&x)[E], const float (&y)[E]) {
  if (!p.rotated) return;
  if (pairing == 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 t = cs[p.pair + e];
      // first of its pair: a c - b s; second: a s + b c
      const float by = y[e] * t.y, xc = x[e] * t.x;
      x[e] = p.first ? fmaf(x[e], t.x, -by) : fmaf(y[e], t.y, xc);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 t = cs[p.pair + (e >> 1)];
      rotate_pair(x[e], x[e + 1], t.x, t.y);
    }
  }
}

template <typename R, int E>
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = Elem<R>::get(v, e);
}

// E values stored in type T (16 bytes, 8 for fp8), rounded to nearest even
template <typename T, int E>
__device__ __forceinline__ void store_values(T* dst, const float (&x)[E]) {
  uint32_t w[4];
  if constexpr (std::is_same<T, uint16_t>::value) {
#pragma unroll
    for (int e = 0; e < E; e += 2) w[e / 2] = pack_bf16_rne(x[e], x[e + 1]);
  } else {
    pack_words<T, E>(x, w);
  }
  if constexpr (E * sizeof(T) == 16)
    st16s(dst, make_uint4(w[0], w[1], w[2], w[3]));
  else
    __builtin_nontemporal_store((u32x2){w[0], w[1]}, reinterpret_cast<u32x2*>(dst));
}

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}
// the sum over N consecutive lanes (8, 16, 32 or 64), in all of them
template <int N>
__device__ __forceinline__ float sum_lanes(float x) {
  x = add_dpp<0xB1>(x);                              // quad_perm [1, 0, 3, 2]
  x = add_dpp<0x4E>(x);                              // quad_perm [2, 3, 0, 1]
  x = add_dpp<0x141>(x);                             // row_half_mirror: the other quad of eight lanes
  if constexpr (N >= 16) x = add_dpp<0x140>(x);      // row_mirror: the other eight of a row
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (N >= 64) {
    const float2 h = halves32(x);
    x = h.x + h.y;
  }
  return x;
}

// Steps (of rs heads) of a workgroup, so that a small call's heads are spread over several.
//
// Workgroups below which they are: not at all, up to 256, up to 1,024 workgroups: 16 tokens 8.8, 5.1, 5.2 us, 8 layers of them -,
// 6.8, 6.0; 300 tokens of 48 heads rotated -, 4.6, 4.0.
constexpr int64_t kSmallGrid = 1024;
inline int steps_per_block(int64_t blocks, int rows, int rs) {
  const int steps = (rows + rs - 1) / rs;
  const int64_t want = (kSmallGrid + blocks - 1) / blocks;         // workgroups a token
  return (int)((steps + (want < steps ? want : steps) - 1) / (want < steps ? want : steps));
}

}  // namespace

}  // namespace kvg
