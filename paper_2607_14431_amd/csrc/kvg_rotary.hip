// Rotary positions of packed rows, alone (kvg_rotate) and with the heads' norms and the append to the
// paged cache (kvg_norm_append).
//
// One workgroup per token (and group of layers).  Angles pos * theta_i, their cosines and sines are taken in fp64
// once per token and kept in LDS as fp32; then every 16-byte vector of the token's heads is a lane's work: a head
// is D / E consecutive lanes (E values a vector), which sum its squares among themselves for the norm.  A vector
// whose pair lies in another one (half pairing) reads that one too, from L1.
#include "kvg_launch.h"
#include "kvg_packed.h"

#include <type_traits>

namespace kvg {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint4 ld16(const void* p) { return *reinterpret_cast<const uint4*>(p); }

// cos and sin of pos * theta_i, times the amplitude, for i < dim / 2
__device__ __forceinline__ void fill_table(const RotaryArgs& r, int64_t pos, float2* cs) {
  for (int p = threadIdx.x; p < r.dim / 2; p += blockDim.x) {
    double s, c;
    sincos((double)pos * r.theta[p], &s, &c);
    cs[p] = make_float2((float)(c * r.amplitude), (float)(s * r.amplitude));
  }
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

// x: the vector's values, y: its partners' (half pairing)
template <int E>
__device__ __forceinline__ void rotate_values(const Place& p, int pairing, const float2* cs, float (&x)[E], const float (&y)[E]) {
  if (!p.rotated) return;
  if (pairing == 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 t = cs[p.pair + e];
      float a = p.first ? x[e] : y[e], b = p.first ? y[e] : x[e];
      rotate_pair(a, b, t.x, t.y);
      x[e] = p.first ? a : b;
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

// E values stored in type T (16 bytes, 8 for fp8)
template <typename T, int E>
__device__ __forceinline__ void store_values(T* dst, const float (&x)[E]) {
  uint32_t w[4];
  pack_words<T, E>(x, w);
  if constexpr (E * sizeof(T) == 16)
    *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  else
    *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
}

template <typename R>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
  constexpr int E = Elem<R>::kPerVec;
  __shared__ float2 cs[kMaxHalfDim];
  const int64_t tok = blockIdx.x;
  fill_table(a.rot, a.positions[tok], cs);
  __syncthreads();
  const int vecs = a.D / E;
  const R* x = reinterpret_cast<const R*>(a.x) + tok * a.x_stride;
  R* y = reinterpret_cast<R*>(a.y) + tok * a.y_stride;
  // a head's lanes are in one wave, so a row rotated in place is read whole before it is written
  for (int it = threadIdx.x; it < a.n_heads * vecs; it += kThreads) {
    const int e0 = (it % vecs) * E;
    const int64_t head = (int64_t)(it / vecs) * a.D;
    const Place p = place(a.rot, e0);
    const uint4 own = ld16(x + head + e0), other = ld16(x + head + p.partner);
    float v[E], w[E];
    unpack<R>(own, v);
    unpack<R>(other, w);
    rotate_values(p, a.rot.pairing, cs, v, w);
    if (p.rotated) {
      store_values<R>(y + head + e0, v);
    } else {
      *reinterpret_cast<uint4*>(y + head + e0) = own;
    }
  }
}

// T: cache storage.  A wave's 64 lanes look for the token's sequence together.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_append_kernel(const NormAppendArgs a) {
  using R = typename RawOf<T>::type;
  constexpr int E = Elem<R>::kPerVec;
  __shared__ float2 cs[kMaxHalfDim];
  const int tok = blockIdx.x;
  const int lane = threadIdx.x & 63;
  int b = -1;
  for (int b0 = 0; b0 < a.seqs.batch; b0 += 64) {
    const int i = b0 + lane;
    const bool after = i < a.seqs.batch && a.seqs.cu[i + 1] > tok;
    const uint64_t m = __builtin_amdgcn_ballot_w64(after);
    if (m != 0) {
      b = b0 + __builtin_ctzll(m);
      break;
    }
  }
  if (b < 0) return;                                      // behind the last sequence (uniform)
  const SeqRange s = seq_range(a.seqs, b);
  const int i = tok - s.row0;
  if (i < 0 || i >= s.len) return;
  const int t = s.ctx + i;
  const int32_t page = a.seqs.tables[(int64_t)b * a.seqs.max_pages + t / kPage];
  const bool page_ok = page >= 0 && page < a.n_pages;
  fill_table(a.rot, a.start_pos[b] + t, cs);
  __syncthreads();

  const int D = a.D, vecs = D / E;
  const int n_q = a.q_raw != nullptr ? a.Hq : 0;
  const int l_end = min((int)(blockIdx.y + 1) * a.layers_per_block, a.n_layers);
  for (int l = blockIdx.y * a.layers_per_block; l < l_end; ++l) {
    const int64_t row = (int64_t)l * a.seqs.n_tokens + tok;
    const R* q = reinterpret_cast<const R*>(a.q_raw) + row * a.q_stride;
    const R* k = reinterpret_cast<const R*>(a.k_raw) + row * a.k_stride;
    const R* v = reinterpret_cast<const R*>(a.v_raw) + row * a.v_stride;
    const int64_t pool = (int64_t)(a.layer0 + l) * a.layer_elems + ((int64_t)page * a.Hkv * kPage + t % kPage) * D;
    for (int it = threadIdx.x; it < (n_q + 2 * a.Hkv) * vecs; it += kThreads) {
      const int h = it / vecs, e0 = (it - h * vecs) * E;
      if (h >= n_q + a.Hkv) {                             // values
        const int g = h - n_q - a.Hkv;
        const uint4 raw = ld16(v + (int64_t)g * D + e0);
        if (!page_ok) continue;
        T* dst = reinterpret_cast<T*>(a.v_pool) + pool + (int64_t)g * kPage * D + e0;
        if constexpr (std::is_same<T, R>::value) {
          *reinterpret_cast<uint4*>(dst) = raw;
        } else {
          float x[E];
          unpack<R>(raw, x);
          store_values<T>(dst, x);
        }
        continue;
      }
      const bool is_q = h < n_q;
      const int g = is_q ? h : h - n_q;
      const R* src = (is_q ? q : k) + (int64_t)g * D;
      const Place p = place(a.rot, e0);
      float x[E], y[E];
      unpack<R>(ld16(src + e0), x);
      unpack<R>(ld16(src + p.partner), y);
      const void* wp = is_q ? a.q_weight : a.k_weight;
      if (wp != nullptr) {
        const R* w = reinterpret_cast<const R*>(wp) + (int64_t)l * D;
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum = fmaf(x[e], x[e], sum);
        for (int m = 1; m < vecs; m <<= 1) sum += __shfl_xor(sum, m);
        const float inv = 1.0f / sqrtf(sum / (float)D + a.eps);
        float wx[E], wy[E];
        unpack<R>(ld16(w + e0), wx);
        unpack<R>(ld16(w + p.partner), wy);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x[e] = x[e] * inv * (wx[e] + a.weight_offset);
          y[e] = y[e] * inv * (wy[e] + a.weight_offset);
        }
      }
      rotate_values(p, a.rot.pairing, cs, x, y);
      if (is_q) {
        store_values<R>(reinterpret_cast<R*>(a.q_out) + (row * a.Hq + g) * D + e0, x);
      } else if (page_ok) {
        store_values<T>(reinterpret_cast<T*>(a.k_pool) + pool + (int64_t)g * kPage * D + e0, x);
      }
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int dtype, hipStream_t stream) {
  if (dtype == kDtypeF32)
    rotate_kernel<float><<<a.n_tokens, kThreads, 0, stream>>>(a);
  else
    rotate_kernel<uint16_t><<<a.n_tokens, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_norm_append(const NormAppendArgs& args, int dtype, hipStream_t stream) {
  NormAppendArgs a = args;
  // layers per workgroup: enough workgroups to fill the chip, fewer sincos recomputations
  const int64_t per = ((int64_t)a.n_layers * a.seqs.n_tokens + 8191) / 8192;
  a.layers_per_block = (int)(per < 1 ? 1 : per > a.n_layers ? a.n_layers : per);
  if (a.layers_per_block < (a.n_layers + 65534) / 65535) a.layers_per_block = (a.n_layers + 65534) / 65535;
  const dim3 grid(a.seqs.n_tokens, (a.n_layers + a.layers_per_block - 1) / a.layers_per_block);
  switch (dtype) {
    case kDtypeF32: norm_append_kernel<float><<<grid, kThreads, 0, stream>>>(a); break;
    case kDtypeBf16: norm_append_kernel<uint16_t><<<grid, kThreads, 0, stream>>>(a); break;
    case kDtypeFp8: norm_append_kernel<uint8_t><<<grid, kThreads, 0, stream>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace kvg
