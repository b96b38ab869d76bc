// Norm, rotation and append of packed sequences to a cache of 8-bit integers (kvg_int8_append), and the scales of blocks.
//
// A page's rows share a scale, so the unit of work is a page that the call's tokens fall into: a workgroup takes it for a group of
// layers and heads, and a wave a (layer, KV head) of it at a time, up to 16 rows of keys or of values held in registers:
//   x = the new rows, normed and rotated, fp32;  s = max(max |x| / 127, scale before);  n = rint(x / s)
// and where the page held rows and s grew, their integers n <- rint(n * before / s).  Query heads of the page's tokens are
// waves' work too.  The rotation of the page's tokens is computed once (fp64 angles, fp32 cosines and sines in LDS).
//
// Bound: 14,100 tokens of 32 + 2 x 16 heads x 128 take 101 us (406 MB, 4.0 TB/s), the vector unit busy for 62 of them: 21 instructions
// for 64 values, of which the norm has nine, the rotation five and the integers three (with a clamp, a conversion and shifts for each
// integer it was eight, and 108 us).  One to six workgroups a page take 100 to 103 us, eight 111; 16 single tokens of 16 + 2 x 8 heads x
// 256, a page each, 7 us with a wave for every head, 18 with four for all: metadata, the fp64 angles behind their barrier, and only then
// the raw rows, head after head (kvg_rotary.hip requests its first rows before the angles, this kernel does not).
#include "kvg_int8.h"
#include "kvg_launch.h"
#include "kvg_rotary.h"

#include <math.h>

namespace kvg {

namespace {

constexpr int kThreads = 256;

// Eight values times inv, rounded to integers, as bytes.  |x inv| <= 127 but for a few last bits, so 1.5 2^23 added to it rounds it to
// the nearest even and leaves the integer in the low byte.
__device__ __forceinline__ u32x2 to_int8(const float (&x)[8], float inv) {
#pragma clang fp contract(off)
  constexpr float kRound = 12582912.0f;
  uint32_t n[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) n[e] = __float_as_uint(x[e] * inv + kRound);
  auto four = [&](int e) -> uint32_t {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(n[e + 3], n[e + 2], 0x0C0C0400u), __builtin_amdgcn_perm(n[e + 1], n[e], 0x0C0C0400u), 0x05040100u);
  };
  return (u32x2){four(0), four(4)};
}

// A page's cosines and sines: a lane's eight pairs lie 80 bytes from its neighbour's, so that a wave's 16-byte reads meet all banks
// alike (64 bytes apart, half the reads' time was conflicts).
constexpr int turn_at(int pair) { return pair + pair / 8 * 2; }

// y: the values of this lane's partners (half pairing).  Where all of a head turns they are half a head's lanes away.
template <int D>
__device__ __forceinline__ void partners(const Place& p, bool whole, int e0, const float (&x)[8], float (&y)[8]) {
  if (D == 64 || !whole) {
    from_partner<8>(p, e0, x, y);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (D == 128) {
      y[e] = __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x[e]), 0x128, 0xF, 0xF, true));      // rows of 16 by 8
    } else {
      const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[e]), __float_as_uint(x[e]), false, false);
      y[e] = __uint_as_float(threadIdx.x & 16 ? both[0] : both[1]);
    }
  }
}

template <int D, typename Axes>
__global__ __launch_bounds__(kThreads) void int8_append_kernel(const NormAppendArgs a, const Int8Scales scales, const Axes axes) {
  constexpr int VECS = D / 8, RPP = 64 / VECS, NP = kPage / RPP;      // lanes of a row, rows at a time, times
  __shared__ __attribute__((aligned(16))) float2 cs[kPage][turn_at(D / 2)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int e0 = lane % VECS * 8, r0 = lane / VECS;
  const Place p = place(a.rot, e0);

  const SeqUnit u = find_unit(a.seqs, (int)blockIdx.x, [](const SeqRange& s) {
    return s.len > 0 ? (s.ctx + s.len - 1) / kPage - s.ctx / kPage + 1 : 0;
  });
  if (u.b < 0) return;
  const int slot0 = u.range.ctx / kPage + u.at;                        // the page's place in the sequence
  const int t0 = max(u.range.ctx, slot0 * kPage), t1 = min(u.range.ctx + u.range.len, (slot0 + 1) * kPage);
  const int held = t0 - slot0 * kPage, n = t1 - t0;                    // rows before, new rows
  const int64_t tok0 = u.range.row0 + (t0 - u.range.ctx);              // first packed row
  const int32_t page = a.seqs.tables[(int64_t)u.b * a.seqs.max_pages + slot0];
  const bool page_ok = page >= 0 && page < a.n_pages;
  int64_t pos0 = 0;
  if constexpr (std::is_same<Axes, NoAxes>::value) pos0 = a.start_pos[u.b] + t0;
  const int half = a.rot.dim / 2;
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int r = i / half, j = i % half;
    cs[r][turn_at(j)] = turn(a.rot, pair_position(axes, pos0 + r, tok0 + r, a.seqs.n_tokens, j), j);
  }
  __syncthreads();

  const int n_q = a.q_raw != nullptr ? a.Hq : 0, heads = n_q + 2 * a.Hkv;
  const int h_end = min(heads, (int)(blockIdx.z + 1) * a.steps);
  const int l_end = min(a.n_layers, (int)(blockIdx.y + 1) * a.layers_per_block);
  for (int l = blockIdx.y * a.layers_per_block; l < l_end; ++l) {
    const int64_t row_l = (int64_t)l * a.seqs.n_tokens + tok0;
    for (int h = blockIdx.z * a.steps + wave; h < h_end; h += kThreads / 64) {
      const bool is_q = h < n_q, is_k = !is_q && h < n_q + a.Hkv;
      const int head = is_q ? h : is_k ? h - n_q : h - n_q - a.Hkv;
      if (!is_q && !page_ok) continue;
      const uint16_t* src = is_q   ? static_cast<const uint16_t*>(a.q_raw) + row_l * a.q_stride
                            : is_k ? static_cast<const uint16_t*>(a.k_raw) + row_l * a.k_stride
                                   : static_cast<const uint16_t*>(a.v_raw) + row_l * a.v_stride;
      const int64_t stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
      src += (int64_t)head * D + e0;
      uint4 raw[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int r = i * RPP + r0;
        raw[i] = make_uint4(0, 0, 0, 0);
        if (r < n) raw[i] = *reinterpret_cast<const uint4*>(src + r * stride);
      }
      // where the page's integers and scale lie
      const int64_t lp = ((int64_t)(a.layer0 + l) * a.n_pages + page) * a.Hkv + head;
      int8_t* slab = static_cast<int8_t*>(is_k ? a.k_pool : a.v_pool) + lp * (kPage * D) + e0;
      float* scale_at = (is_k ? scales.k : scales.v) + lp;
      const float before = !is_q && held > 0 ? *scale_at : 0.0f;
      const uint16_t* weight = static_cast<const uint16_t*>(is_q ? a.q_weight : is_k ? a.k_weight : nullptr);
      float w[8];
      if (weight != nullptr) {
        unpack<uint16_t>(*reinterpret_cast<const uint4*>(weight + (int64_t)l * D + e0), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] += a.weight_offset;
      }
      float x[NP][8];
      uint32_t most = 0;                                               // largest |x| as bits: Inf and NaN above all others
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if (i * RPP >= n) {                                            // no such rows (uniform)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
          continue;
        }
        unpack<uint16_t>(raw[i], x[i]);
        if (weight != nullptr) {
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = fmaf(x[i][e], x[i][e], sum);
          const float inv = 1.0f / sqrtf(sum_lanes<VECS>(sum) * (1.0f / D) + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * inv * w[e];
        }
        if (is_q || is_k) {
          float y[8];
          if (a.rot.pairing == 0) partners<D>(p, a.rot.dim == D, e0, x[i], y);
          rotate_values(p, a.rot.pairing, cs[min(i * RPP + r0, n - 1)] + (turn_at(p.pair) - p.pair), x[i], y);
        }
        if (is_q) {
          const int r = i * RPP + r0;
          if (r < n) store_values<uint16_t>(static_cast<uint16_t*>(a.q_out) + ((row_l + r) * a.Hq + head) * D + e0, x[i]);
        } else if (i * RPP + r0 < n) {
#pragma unroll
          for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[i][e]) & 0x7FFFFFFFu);
        }
      }
      if (is_q) continue;
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, m));
      // a block with an Inf or NaN, now or before, has scale NaN
      const bool bad = most >= 0x7F800000u || !(before < INFINITY);
      const float now = most == 0 ? 0.0f : fmaxf(__uint_as_float(most) / kInt8Max, kInt8Least);
      const float scale = bad ? __uint_as_float(0x7FC00000u) : fmaxf(now, before);
      const float inv = bad || scale == 0.0f ? 0.0f : 1.0f / scale;
      if (held > 0 && !bad && scale > before) {
        const float ratio = before / scale;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int r = i * RPP + r0;
          if (r >= held) continue;
          u32x2* at = reinterpret_cast<u32x2*>(slab + r * D);
          const u32x2 old = *at;
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = (float)(int8_t)(old[e / 4] >> (8 * (e % 4)));
          *at = to_int8(y, ratio);
        }
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int r = i * RPP + r0;
        if (r < n) *reinterpret_cast<u32x2*>(slab + (held + r) * D) = bad ? (u32x2){0, 0} : to_int8(x[i], inv);
      }
      if (lane == 0) *scale_at = scale;
    }
  }
}

template <int D, typename Axes>
hipError_t launch_append_d(NormAppendArgs a, const Int8Scales& s, const Axes& axes, hipStream_t stream) {
  const int64_t units = int8_append_units(a.seqs);
  const int heads = (a.q_raw != nullptr ? a.Hq : 0) + 2 * a.Hkv;
  const int64_t per = ((int64_t)a.n_layers * units + 4095) / 4096;
  a.layers_per_block = (int)(per < 1 ? 1 : per > a.n_layers ? a.n_layers : per);
  if (a.layers_per_block < (a.n_layers + 65534) / 65535) a.layers_per_block = (a.n_layers + 65534) / 65535;
  const unsigned layer_groups = (a.n_layers + a.layers_per_block - 1) / a.layers_per_block;
  a.steps = 4 * steps_per_block(units * layer_groups, heads, 4);
  const dim3 grid((unsigned)units, layer_groups, (heads + a.steps - 1) / a.steps);
  int8_append_kernel<D, Axes><<<grid, kThreads, 0, stream>>>(a, s, axes);
  return hipGetLastError();
}

template <typename Axes>
hipError_t launch_append(const NormAppendArgs& a, const Int8Scales& s, const Axes& axes, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_append_d<64>(a, s, axes, stream);
    case 128: return launch_append_d<128>(a, s, axes, stream);
    case 256: return launch_append_d<256>(a, s, axes, stream);
    default: return hipErrorInvalidValue;
  }
}

// A lane a scale.
template <bool kDeposit>
__global__ __launch_bounds__(kThreads) void int8_scales_kernel(const Int8ScaleCopyArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= int8_scale_values(a)) return;
  const int h = (int)(i % a.Hkv);
  const int64_t rest = i / a.Hkv;
  const int p = (int)(rest % a.n_block_pages), kv = (int)(rest / a.n_block_pages % 2), l = (int)(rest / a.n_block_pages / 2);
  const int32_t page = a.block_table[a.first_page + p];
  const bool ok = page >= 0 && page < a.n_pages;
  float* at = (kv ? a.scales.v : a.scales.k) + ((int64_t)l * a.n_pages + (ok ? page : 0)) * a.Hkv + h;
  if constexpr (kDeposit)
    a.payload[i] = ok ? *at : 0.0f;
  else if (ok)
    *at = a.payload[i];
}

}  // namespace

hipError_t launch_int8_append(const NormAppendArgs& a, const Int8Scales& s, const AxesArgs* axes, hipStream_t stream) {
  return axes != nullptr ? launch_append(a, s, *axes, stream) : launch_append(a, s, NoAxes{}, stream);
}

hipError_t launch_int8_scales(const Int8ScaleCopyArgs& a, bool deposit, hipStream_t stream) {
  const unsigned grid = (unsigned)((int8_scale_values(a) + kThreads - 1) / kThreads);
  if (deposit)
    int8_scales_kernel<true><<<grid, kThreads, 0, stream>>>(a);
  else
    int8_scales_kernel<false><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace kvg
