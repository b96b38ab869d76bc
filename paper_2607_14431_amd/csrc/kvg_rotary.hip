// Rotary positions of packed rows, alone (kvg_rotate) and with the heads' norms and the append to the
// paged cache (kvg_norm_append).
//
// A workgroup takes a token (in a small call a part of its heads, in a large one several layers).  Angles pos * theta_i,
// their cosines and sines are taken in fp64 once per token and kept in LDS as fp32; then every 16-byte vector of the
// token's heads is a lane's work: a head is D / E consecutive lanes (E values a vector), which sum its squares among
// themselves for the norm (DPP and half swaps) and give each other the partners of half pairing (ds_bpermute).  A lane
// keeps its place in the head, and with it its weights, from head to head.
//
// What bounds them: HBM in large calls, where each raw value is read and each result written once (eight prompts up to 4,096
// tokens, 32 + 2 x 16 heads x 128: 101 us, 4.7 TB/s, and 78 to 90 when the last-level cache holds inputs and pages of a repeated
// call; a 4,096-token block of 48 heads x 128 rotated: 16.5 us, 6.1 TB/s); the round
// trips in small ones (metadata, then angles; the first rows are requested before either: 16 single tokens of 16 + 2 x 8
// heads x 256 5 to 6 us, one token's 24 heads rotated in 3.0).  Partners read from memory cost their second load and the registers
// of two waves a SIMD (those prompts 89 us; fp8, 1,063 tokens x 6 layers 40, then 34).  Four tokens a workgroup, whose tables fill all
// lanes, were no faster (45 us, then 41), nor more wavefronts with spills (seven a SIMD: 81 us for the prompts, 37; eight: 140, 52).
#include "kvg_launch.h"
#include "kvg_mfma.h"
#include "kvg_packed.h"

#include <type_traits>

namespace kvg {

namespace {

constexpr int kThreads = 256;
// Workgroups below which a token's heads are spread over several: not at all, up to 256, up to 1,024 workgroups: 16 tokens 8.8, 5.1,
// 5.2 us, 8 layers of them -, 6.8, 6.0; 300 tokens of 48 heads rotated -, 4.6, 4.0.
constexpr int64_t kSmallGrid = 1024;

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

template <typename R, int D>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
  constexpr int E = Elem<R>::kPerVec, VECS = D / E, RS = kThreads / VECS;      // RS: heads at a time
  __shared__ float2 cs[kMaxHalfDim];
  const int64_t tok = blockIdx.x;
  const int e0 = threadIdx.x % VECS * E;
  const Place p = place(a.rot, e0);
  const R* x = reinterpret_cast<const R*>(a.x) + tok * a.x_stride;
  R* y = reinterpret_cast<R*>(a.y) + tok * a.y_stride;
  int h = blockIdx.y * RS * a.steps + threadIdx.x / VECS;
  const int h_end = min(a.n_heads, (int)(blockIdx.y + 1) * RS * a.steps);
  uint4 own = make_uint4(0, 0, 0, 0);
  auto load = [&](int head) {
    if (head < h_end) own = ld16(x + (int64_t)head * D + e0);
  };
  load(h);                                           // before the angles, which wait for the position
  const int64_t pos = a.positions[tok];
  for (int i = threadIdx.x; i < a.rot.dim / 2; i += kThreads) cs[i] = turn(a.rot, pos, i);
  __syncthreads();
  // a head's lanes are in one wave, so a row rotated in place is read whole before it is written
  for (; h < h_end; h += RS) {
    float v[E], w[E];
    const uint4 raw = own;
    load(h + RS);
    unpack<R>(raw, v);
    if (a.rot.pairing == 0) from_partner<E>(p, e0, v, w);
    rotate_values(p, a.rot.pairing, cs, v, w);
    if (p.rotated)
      store_values<R>(y + (int64_t)h * D + e0, v);
    else
      st16s(y + (int64_t)h * D + e0, raw);
  }
}

// T: cache storage.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void norm_append_kernel(const NormAppendArgs a) {
  using R = typename RawOf<T>::type;
  constexpr int E = Elem<R>::kPerVec, VECS = D / E, RS = kThreads / VECS;      // RS: heads at a time
  __shared__ float2 cs[kMaxHalfDim];

  const int tok = blockIdx.x;
  const int n_q = a.q_raw != nullptr ? a.Hq : 0, rows = n_q + 2 * a.Hkv;
  const int e0 = threadIdx.x % VECS * E;
  const Place p = place(a.rot, e0);
  const int l_begin = blockIdx.y * a.layers_per_block, l_end = min(l_begin + a.layers_per_block, a.n_layers);
  const int r_begin = blockIdx.z * RS * a.steps + threadIdx.x / VECS, r_end = min(rows, (int)(blockIdx.z + 1) * RS * a.steps);

  // row r of the token: its queries, then its keys, then its values
  uint4 own = make_uint4(0, 0, 0, 0);
  auto load = [&](int l, int r) {
    if (r >= r_end) return;
    const int64_t at = (int64_t)l * a.seqs.n_tokens + tok;
    const R* s = r < n_q           ? reinterpret_cast<const R*>(a.q_raw) + at * a.q_stride + (int64_t)r * D
                 : r < n_q + a.Hkv ? reinterpret_cast<const R*>(a.k_raw) + at * a.k_stride + (int64_t)(r - n_q) * D
                                   : reinterpret_cast<const R*>(a.v_raw) + at * a.v_stride + (int64_t)(r - n_q - a.Hkv) * D;
    own = ld16(s + e0);
  };
  load(l_begin, r_begin);                            // before the sequence and the angles are known

  const SeqUnit u = find_token(a.seqs, tok);
  if (u.b < 0) return;                               // a row of no sequence (uniform)
  const int t = u.range.ctx + u.at;
  const int32_t page = a.seqs.tables[(int64_t)u.b * a.seqs.max_pages + t / kPage];
  const bool page_ok = page >= 0 && page < a.n_pages;
  const int64_t row = (int64_t)page * a.Hkv * kPage + t % kPage;       // of the token in its (page, head 0) slab
  const int64_t pos = a.start_pos[u.b] + t;
  for (int i = threadIdx.x; i < a.rot.dim / 2; i += kThreads) cs[i] = turn(a.rot, pos, i);
  __syncthreads();

  for (int l = l_begin; l < l_end; ++l) {
    // this lane's weights
    const R* wq = reinterpret_cast<const R*>(a.q_weight) + (int64_t)l * D;
    const R* wk = reinterpret_cast<const R*>(a.k_weight) + (int64_t)l * D;
    uint4 wq_own, wk_own;
    if (a.q_weight != nullptr) wq_own = ld16(wq + e0);
    if (a.k_weight != nullptr) wk_own = ld16(wk + e0);
    T* kpool = reinterpret_cast<T*>(a.k_pool) + (int64_t)(a.layer0 + l) * a.layer_elems;
    T* vpool = reinterpret_cast<T*>(a.v_pool) + (int64_t)(a.layer0 + l) * a.layer_elems;
#pragma unroll 1
    for (int r = r_begin; r < r_end; r += RS) {
      const uint4 raw = own;
      if (r + RS < r_end)
        load(l, r + RS);
      else if (l + 1 < l_end)
        load(l + 1, r_begin);
      if (r >= n_q + a.Hkv) {                        // values
        T* dst = vpool + (row + (int64_t)(r - n_q - a.Hkv) * kPage) * D + e0;
        if (!page_ok) continue;
        if constexpr (std::is_same<T, R>::value) {
          st16s(dst, raw);
        } else {
          float x[E];
          unpack<R>(raw, x);
          store_values<T>(dst, x);
        }
        continue;
      }
      const bool is_q = r < n_q;
      float x[E], y[E];
      unpack<R>(raw, x);
      if ((is_q ? a.q_weight : a.k_weight) != nullptr) {
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum = fmaf(x[e], x[e], sum);
        const float inv = 1.0f / sqrtf(sum_lanes<VECS>(sum) * (1.0f / D) + a.eps);
        float wx[E];
        unpack<R>(is_q ? wq_own : wk_own, wx);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = x[e] * inv * (wx[e] + a.weight_offset);
      }
      if (a.rot.pairing == 0) from_partner<E>(p, e0, x, y);
      rotate_values(p, a.rot.pairing, cs, x, y);
      if (is_q) {
        store_values<R>(reinterpret_cast<R*>(a.q_out) + (((int64_t)l * a.seqs.n_tokens + tok) * a.Hq + r) * D + e0, x);
      } else if (page_ok) {
        store_values<T>(kpool + (row + (int64_t)(r - n_q) * kPage) * D + e0, x);
      }
    }
  }
}

// Steps (of RS heads) of a workgroup, so that a small call's heads are spread over several.
int steps_per_block(int64_t blocks, int rows, int rs) {
  const int steps = (rows + rs - 1) / rs;
  const int64_t want = (kSmallGrid + blocks - 1) / blocks;         // workgroups a token
  return (int)((steps + (want < steps ? want : steps) - 1) / (want < steps ? want : steps));
}

template <typename R, int D>
hipError_t launch_rotate_d(RotateArgs a, hipStream_t stream) {
  constexpr int RS = kThreads / (D / Elem<R>::kPerVec);
  a.steps = steps_per_block(a.n_tokens, a.n_heads, RS);
  const dim3 grid(a.n_tokens, (a.n_heads + RS * a.steps - 1) / (RS * a.steps));
  rotate_kernel<R, D><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename R>
hipError_t launch_rotate_t(const RotateArgs& a, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_rotate_d<R, 64>(a, stream);
    case 128: return launch_rotate_d<R, 128>(a, stream);
    case 256: return launch_rotate_d<R, 256>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

template <typename T, int D>
hipError_t launch_norm_append_d(NormAppendArgs a, hipStream_t stream) {
  constexpr int RS = kThreads / (D / Elem<typename RawOf<T>::type>::kPerVec);
  const int rows = (a.q_raw != nullptr ? a.Hq : 0) + 2 * a.Hkv;
  // Layers per workgroup, which share its angles, as long as there are 4,096 workgroups.  One layer each / 4,096 / 2,048
  // workgroups, us: fp8, 1,063 tokens x 6 layers 41.7 / 39.6 / 37.8, x 24 188 / 163 / 179; 14,472 tokens x 4 491 / 414 / 407.
  const int64_t per = ((int64_t)a.n_layers * a.seqs.n_tokens + 4095) / 4096;
  a.layers_per_block = (int)(per < 1 ? 1 : per > a.n_layers ? a.n_layers : per);
  if (a.layers_per_block < (a.n_layers + 65534) / 65535) a.layers_per_block = (a.n_layers + 65534) / 65535;
  const unsigned layer_groups = (a.n_layers + a.layers_per_block - 1) / a.layers_per_block;
  a.steps = steps_per_block((int64_t)a.seqs.n_tokens * layer_groups, rows, RS);
  const dim3 grid(a.seqs.n_tokens, layer_groups, (rows + RS * a.steps - 1) / (RS * a.steps));
  norm_append_kernel<T, D><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_append_t(const NormAppendArgs& a, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_norm_append_d<T, 64>(a, stream);
    case 128: return launch_norm_append_d<T, 128>(a, stream);
    case 256: return launch_norm_append_d<T, 256>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int dtype, hipStream_t stream) {
  return dtype == kDtypeF32 ? launch_rotate_t<float>(a, stream) : launch_rotate_t<uint16_t>(a, stream);
}

hipError_t launch_norm_append(const NormAppendArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case kDtypeF32: return launch_norm_append_t<float>(a, stream);
    case kDtypeBf16: return launch_norm_append_t<uint16_t>(a, stream);
    case kDtypeFp8: return launch_norm_append_t<uint8_t>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvg
