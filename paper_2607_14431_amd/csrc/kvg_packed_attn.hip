// Causal attention of packed sequences over the paged cache.
//
// A wave takes one (token, query head): 64 keys at a time, a key per lane for the scores and a few dimensions per
// lane for the weighted values, with a running reference and sum per row.  Keys a row does not see are not read.
#include "kvg_launch.h"
#include "kvg_packed.h"
#include "kvg_rows.h"

#include <math.h>

namespace kvg {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_value(const float* p) { return *p; }
__device__ __forceinline__ float load_value(const uint16_t* p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ float load_value(const uint8_t* p) { return Elem<uint8_t>::get(make_uint4(*p, 0, 0, 0), 0); }
__device__ __forceinline__ void store_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_value(uint16_t* p, float x) { *p = (uint16_t)f32_to_bf16_bits(x); }

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void packed_rows_kernel(const PackedAttnArgs a) {
  using R = typename RawOf<T>::type;
  constexpr int E = Elem<T>::kPerVec;
  constexpr int ER = Elem<R>::kPerVec;
  constexpr int W = kThreads / 64;
  __shared__ float s_q[W][D];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * W + wave;
  if (id >= (int64_t)a.n_layers * a.seqs.n_tokens * a.Hq) return;
  const int h = (int)(id % a.Hq);
  const int tok = (int)(id / a.Hq % a.seqs.n_tokens), l = (int)(id / a.Hq / a.seqs.n_tokens);
  int b = -1;
  for (int b0 = 0; b0 < a.seqs.batch; b0 += 64) {
    const int i = b0 + lane;
    const uint64_t m = __builtin_amdgcn_ballot_w64(i < a.seqs.batch && a.seqs.cu[i + 1] > tok);
    if (m != 0) {
      b = b0 + __builtin_ctzll(m);
      break;
    }
  }
  if (b < 0) return;
  const SeqRange s = seq_range(a.seqs, b);
  if (tok < s.row0 || tok >= s.row0 + s.len) return;
  const int n_keys = s.ctx + tok - s.row0 + 1;
  const int lo = window_start(layer_window(a, l), n_keys);
  const int g = h / a.group;
  const int64_t row = (int64_t)l * a.seqs.n_tokens + tok;
  const R* q = reinterpret_cast<const R*>(a.q) + row * a.q_stride + (int64_t)h * D;
  if (lane < D / ER) {
    const uint4 v = ld16(q + lane * ER);
#pragma unroll
    for (int e = 0; e < ER; ++e) s_q[wave][lane * ER + e] = Elem<R>::get(v, e);
  }
  __builtin_amdgcn_wave_barrier();
  const int64_t lbase = (int64_t)(a.layer0 + l) * a.layer_elems;
  const T* kpool = reinterpret_cast<const T*>(a.k_pool) + lbase;
  const T* vpool = reinterpret_cast<const T*>(a.v_pool) + lbase;
  const int32_t* bt = a.seqs.tables + (int64_t)b * a.seqs.max_pages;
  auto slab = [&](int key) -> int64_t {
    const int32_t page = bt[key / kPage];
    return (((int64_t)(page >= 0 && page < a.n_pages ? page : 0) * a.Hkv + g) * kPage + key % kPage) * D;
  };
  float m = -INFINITY, sum = 0.0f, acc[D / 64];
#pragma unroll
  for (int x = 0; x < D / 64; ++x) acc[x] = 0.0f;
  for (int c = lo; c < n_keys; c += 64) {
    const int key = c + lane;
    const T* kr = kpool + slab(min(key, n_keys - 1));
    float sc = 0.0f;
    for (int v = 0; v < D / E; ++v) {
      const uint4 kv = ld16(kr + v * E);
#pragma unroll
      for (int e = 0; e < E; ++e) sc = fmaf(s_q[wave][v * E + e], Elem<T>::get(kv, e), sc);
    }
    sc = key < n_keys ? sc * a.scale_log2 : -INFINITY;
    float mx = sc;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) mx = fmaxf(mx, __shfl_xor(mx, x));
    const float m_new = fmaxf(m, mx), f = merge_factor(m, m_new);
    m = m_new;
    float p = key < n_keys ? exp2f(sc - m) : 0.0f;
    sum = sum * f + p;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) acc[x] *= f;
    const int n = min(64, n_keys - c);
    for (int t = 0; t < n; ++t) {
      const float pt = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), t));
      const T* vr = vpool + slab(c + t) + lane * (D / 64);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) acc[x] = fmaf(pt, load_value(vr + x), acc[x]);
    }
  }
#pragma unroll
  for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
  R* out = reinterpret_cast<R*>(a.out) + (row * a.Hq + h) * D + lane * (D / 64);
#pragma unroll
  for (int x = 0; x < D / 64; ++x) {
    store_value(out + x, acc[x] / sum);
  }
}

template <typename T>
hipError_t launch_rows(const PackedAttnArgs& a, hipStream_t stream) {
  const int64_t waves = (int64_t)a.n_layers * a.seqs.n_tokens * a.Hq;
  const dim3 grid((unsigned)((waves + kThreads / 64 - 1) / (kThreads / 64)));
  switch (a.D) {
    case 64: packed_rows_kernel<T, 64><<<grid, kThreads, 0, stream>>>(a); break;
    case 128: packed_rows_kernel<T, 128><<<grid, kThreads, 0, stream>>>(a); break;
    case 256: packed_rows_kernel<T, 256><<<grid, kThreads, 0, stream>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_attn(const PackedAttnArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case kDtypeF32: return launch_rows<float>(a, stream);
    case kDtypeBf16: return launch_rows<uint16_t>(a, stream);
    case kDtypeFp8: return launch_rows<uint8_t>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvg
