// Device helpers of the packed sequences' MFMA attention kernels: references, LDS layout, values that are not finite,
// the fold of segment states.
#pragma once

#include "kvg_mfma.h"
#include "kvg_packed.h"
#include "kvg_rows.h"

#include <math.h>

#include <type_traits>

namespace kvg {

namespace {

// Grid of the references, log2 units.  A coarse one is seldom passed: with 1 / 4 / 16, 12,288 tokens at head_dim 256 take
// 1,324 / 1,301 / 1,158 us (fp8 1,466 / 1,455 / 1,244), and eight prompts at 128 497 / 492 / 472.  Weights reach 2^-16 at the least for the heaviest key of a row,
// far from the limits of fp32 and bf16, which has its exponents.
constexpr float kStep = 16.0f;

// The reference that a largest score (log2 units) asks for.
__device__ __forceinline__ float reference_of(float mx) { return ceilf(mx * (1.0f / kStep)) * kStep; }

// LDS layout of cache rows of RB bytes.  One direct load brings 1 KiB, kRows = 1024 / RB rows, whose 16-byte units its lanes
// may place in any order: units of the same chunk (16 bytes of a row) of consecutive rows lie side by side, so that
// what a fragment read's lanes take is consecutive, and every read of a kernel is one lane base plus a
// constant.  Loads lie 1024 + PAD bytes apart, which spreads the rows of different loads over the banks.
template <int RB, int PAD>
struct Rows {
  static constexpr int kRows = 1024 / RB;
  static constexpr int kLoad = 1024 + PAD;
  static constexpr int kPageLoads = kPage / kRows;
  static constexpr int kPageBytes = kPageLoads * kLoad;
  // byte offset of a row's chunk; with eight rows a load, four rows x two chunks together
  __host__ __device__ static constexpr int at(int row, int chunk) {
    return row / kRows * kLoad + (kRows == 8 ? (chunk / 2 * 2 + row / 4 % 2) * 128 + chunk % 2 * 64 + row % 4 * 16
                                             : (chunk * kRows + row % kRows) * 16);
  }
  // what lane `lane` of a load brings: byte offset in the load's rows
  __device__ static __forceinline__ int source(int lane) {
    if constexpr (kRows == 8)
      return (lane / 8 % 2 * 4 + lane % 4) * RB + (lane / 16 * 2 + lane / 4 % 2) * 16;
    else
      return lane % kRows * RB + lane / kRows * 16;
  }
};
template <int RB> using KRows = Rows<RB, RB == 512 ? 32 : 64>;
template <int RB> using VRows = Rows<RB, RB == 512 ? 128 : 64>;

// A page (16 rows of the pool at `slab`, the first `rows` of them; zeros past them) into LDS.
template <typename R, int POLICY>
__device__ __forceinline__ void load_page(const void* slab, int rows, lds_char* to, int source, int j0 = 0, int j1 = R::kPageLoads) {
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(slab), 0, rows * (1024 / R::kRows), kBufferWord3);
#pragma unroll
  for (int j = j0; j < j1; ++j)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(to + j * R::kLoad), 16, source, 1024 * j, 0, POLICY);
}

__device__ __forceinline__ float load_value(const float* p) { return *p; }
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
template <typename T, typename R>
__device__ __forceinline__ bool finite_page(char* p, int lane) {
  bool any = false;
#pragma unroll 1
  for (int j = 0; j < R::kPageLoads; ++j) {
    T* v = reinterpret_cast<T*>(p + j * R::kLoad + lane * 16);
    if (!bad_values(*reinterpret_cast<const uint4*>(v), T{})) continue;
    any = true;
#pragma unroll 1
    for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
      if (!(fabsf(load_value(v + e)) < INFINITY)) v[e] = 0;
  }
  return __builtin_amdgcn_ballot_w64(any) != 0;
}

__device__ __forceinline__ f32x16 splat(float x) { return (f32x16)(x); }

__device__ __forceinline__ f32x16 mfma32(const uint4& x, const uint4& y, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x), as_bf16x8(y), c, 0, 0, 0);
}

// A fragment as it is read, eight values a lane.  fp8 is widened where it is used: a conversion beside the read would wait
// for it.
template <bool kFp8>
using Fragment = typename std::conditional<kFp8, uint2, uint4>::type;
__device__ __forceinline__ uint4 widen(const uint4& x) { return x; }
__device__ __forceinline__ uint4 widen(const uint2& x) { return widen_fp8x8(x.x, x.y); }

// K fragment of step ss (32 rows x 16 dims; eight values of head_dim for each lane's row) at the lane's base.
template <int RB, bool kFp8>
__device__ __forceinline__ Fragment<kFp8> k_fragment(const lds_char* lane_base, int ss) {
  if constexpr (kFp8) {
    const u32x2 w = *reinterpret_cast<const lds_u32x2*>(lane_base + KRows<RB>::at(0, ss));
    return make_uint2(w.x, w.y);
  } else {
    return __builtin_bit_cast(uint4, *reinterpret_cast<const lds_u32x4*>(lane_base + KRows<RB>::at(0, 2 * ss)));
  }
}
// V^T fragment of 16 rows, dims 32 d .. 32 d + 31.
template <int RB, bool kFp8>
__device__ __forceinline__ Fragment<kFp8> v_fragment(const lds_char* lane_base, int d) {
  if constexpr (kFp8) {
    const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(lane_base + VRows<RB>::at(0, 2 * d)));
    return make_uint2((uint32_t)w.x, (uint32_t)w.y);
  } else {
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lane_base + VRows<RB>::at(0, 4 * d)));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(lane_base + VRows<RB>::at(8, 4 * d)));
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
__device__ __forceinline__ int k_lane_base(int lane) {
  return kFp8 ? KRows<RB>::at(lane & 31, 0) + 8 * (lane >> 5) : KRows<RB>::at(lane & 31, lane >> 5);
}
template <int RB, bool kFp8>
__device__ __forceinline__ int v_lane_base(int lane) {
  const int tr_k = lane & 15, tr_m = lane >> 4;
  return kFp8 ? VRows<RB>::at(4 * (tr_m >> 1) + ((tr_k >> 1) & 3) + 8 * (tr_k >> 3), tr_m & 1) + 8 * (tr_k & 1)
              : VRows<RB>::at((tr_m >> 1) * 4 + (tr_k >> 2), 2 * (tr_m & 1) + ((tr_k & 3) >> 1)) + 8 * (tr_k & 1);
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
// eight weights (a lane's scores of a block, elements 8 h ..) as a bf16 operand, their sum added to psum as rounded.  The
// matrix cores take bf16 beside bf16 values; a weight is off by half a step (2^-8 of it) at most, which moves a row by that
// part of the spread of its values about the result, as its one rounding to bf16 at the end does
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
// A result that takes in a value that is not finite: Inf and Inf of the other sign give NaN, NaN stays.
__device__ __forceinline__ float take_in(float sum, float v) { return fabsf(sum) < INFINITY ? v : sum + v; }

// The values of keys [key0, key1) that are not finite, to those of the pairs [pair0, pair0 + pairs) of a sequence that see them:
// put(pair - pair0, dimension, value), a dimension per lane, the keys in ascending order.  For the keys a kernel has left out; by
// one wave, so that the order is always the same.
template <typename T, typename Put>
__device__ __forceinline__ void put_bad_values(const PackedAttnArgs& a, const T* vpool, const int32_t* table, int g, int key0, int key1,
                                            int W, int ctx, int lg, int pair0, int pairs, Put put) {
  for (int key = key0; key < key1; ++key) {
    const int32_t page = table[key / kPage];
    const T* vr = vpool + (((int64_t)(page >= 0 && page < a.n_pages ? page : 0) * a.Hkv + g) * kPage + key % kPage) * a.D;
    for (int x = __lane_id(); x < a.D; x += 64) {
      const float v = load_value(vr + x);
      if (fabsf(v) < INFINITY) continue;
      for (int p = 0; p < pairs; ++p) {
        const int n = ctx + ((pair0 + p) >> lg);
        if (key <= n && key >= window_start(W, n + 1)) put(p, x, v);
      }
    }
  }
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

// Where a split tile launch leaves its partials: blocks of 32 pairs x D sums for every (layer, tile, KV head, block of the
// tile, segment).  A block's sums are in the order of the matrix steps' results (lane of 64, 4 dims), so that they are
// written and read 1 KiB at a time.
__device__ __forceinline__ int64_t part_block(const PackedAttnArgs& a, int n_seg, int l, int slot, int g, int blocks, int i, int seg) {
  return ((((int64_t)l * a.n_tiles + slot) * a.Hkv + g) * blocks + i) * n_seg + seg;
}
__device__ __forceinline__ int part_at(int pair, int x) { return ((x >> 3) * 64 + ((x >> 2) & 1) * 32 + pair) * 4 + (x & 3); }

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
