// Packed attention of sequences with few rows (single tokens, short chunks): a workgroup per (layer, sequence, KV head,
// segment of kPackedSeg keys), up to kFewPairs (row, query head) pairs, and the fold of segments.
//
// The sums are those of the tile kernel (kvg_packed_mfma.hip), operation for operation: blocks of 32 keys, their
// references and sums one after the other.  What can be done side by side without changing them is: the
// scores of a unit's blocks (a block per wave), then the weights, then the weighted values (a part of
// head_dim per wave, over all of the unit's blocks in order).  Through LDS go the blocks' largest scores,
// the rounded weights (as MFMA operands) and their sums.
//
// What bounds it: HBM in large launches (16 tokens over up to 32k keys, 8 KV heads x 256: 3.24 GB in 521 us, 6.2 TB/s, the bytes
// read are the cached ones), the chain of requests in small ones (16 tokens over 600 keys, 2 KV heads x 128: 17 us, and 4 for the fold).
// K and V of a unit have a buffer each: the next unit's K lands while this one's
// weights and values are worked on, its V during the next unit's scores.
#include "kvg_launch.h"
#include "kvg_packed_mfma.h"

#include <type_traits>

namespace kvg {

namespace {

// s_waitcnt operand that waits for vmcnt <= n alone (gfx9 encoding: bits 3:0 and 15:14)
constexpr int vm_wait(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }
constexpr int kLgkmWait = 0xC07F;      // lgkmcnt(0) alone
constexpr int kStream = 2;             // buffer load policy: nontemporal (every row is read once)

// kWaves: waves of a workgroup, a block of 32 keys and D / kWaves dimensions each
template <typename T, int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void packed_few_kernel(const PackedAttnArgs a) {
  constexpr bool kFp8 = sizeof(T) == 1;
  constexpr int RB = D * (int)sizeof(T), NS = D / 16;
  constexpr int NDW = D / 32 / kWaves;               // 32-wide blocks of head_dim per wave
  constexpr int kUnitKeys = 32 * kWaves;
  using KR = KRows<RB>;
  using VR = VRows<RB>;
  constexpr int kLoads = 2 * KR::kPageLoads;         // direct loads of a wave's block, K or V
  static_assert(D / 32 % kWaves == 0 && kPackedSeg % kUnitKeys == 0, "units");
  __shared__ __attribute__((aligned(1024))) char s_k[2 * kWaves * KR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char s_v[2 * kWaves * VR::kPageBytes];
  __shared__ uint4 s_p[kWaves][2][64];
  __shared__ float s_mx[kWaves][32], s_sum[kWaves][32];
  __shared__ int s_bad;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lrow = lane & 31, half = lane >> 5;
  const int lg = 31 - __builtin_clz(a.group);
  // (layer, sequence, segment, KV head), the KV head fastest: workgroups without work come in runs (see the tile kernel)
  uint32_t id = blockIdx.x;
  const int g = (int)(id % (uint32_t)a.Hkv);
  id /= (uint32_t)a.Hkv;
  int seg = (int)(id % (uint32_t)a.part.n_seg);
  id /= (uint32_t)a.part.n_seg;
  const int b = (int)(id % (uint32_t)a.seqs.batch);
  const int l = (int)(id / (uint32_t)a.seqs.batch);
  seg = (int)((uint32_t)(seg + b) % (uint32_t)a.part.n_seg);
  const int32_t* bt = a.seqs.tables + (int64_t)b * a.seqs.max_pages;
  // page ids of the segment, one per lane (requested with the sequence's range)
  const int32_t pg = bt[min(seg * (kPackedSeg / kPage) + (lane & 31), a.seqs.max_pages - 1)];
  const SeqRange sq = seq_range(a.seqs, b);
  if (sq.len == 0 || !is_few(a, sq)) return;
  const int n_pairs = sq.len << lg;
  const int W = layer_window(a, l);
  const int first_n = sq.ctx, n_hi = sq.ctx + sq.len;        // the first row's index; keys [0, n_hi) are needed
  const int first_lo = window_start(W, first_n + 1), mask_lo = window_start(W, n_hi);
  const int k_end = min(n_hi, (seg + 1) * kPackedSeg);
  const int k_begin = max(seg * kPackedSeg, first_lo & ~(kUnitKeys - 1));
  if (k_begin >= k_end) return;
  const int n_units = (k_end - k_begin + kUnitKeys - 1) / kUnitKeys;

  const int pair = min(lrow, n_pairs - 1);
  const bool pair_ok = lrow < n_pairs;
  const int row = pair >> lg, head = g * a.group + (pair & (a.group - 1));
  const int row_n = sq.ctx + row, row_lo = window_start(W, row_n + 1);

  const int64_t lbase = (int64_t)(a.layer0 + l) * a.layer_elems;
  const T* kpool = reinterpret_cast<const T*>(a.k_pool) + lbase;
  const T* vpool = reinterpret_cast<const T*>(a.v_pool) + lbase;

  // ---- loads of this wave's block of unit u (two pages, K or V); rows from k_end on read as zeros
  const int source = KR::source(lane);               // the same for V
  auto issue = [&](auto rows_type, const T* pool, char* dst, int u) {
    using R = decltype(rows_type);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int key = k_begin + u * kUnitKeys + wave * 32 + p * kPage;
      int32_t page = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_readlane(pg, (key / kPage) & 31));
      page = (page >= 0 && page < a.n_pages) ? page : 0;
      load_page<R, kStream>(pool + ((int64_t)page * a.Hkv + g) * kPage * D, __builtin_amdgcn_readfirstlane(min(max(k_end - key, 0), kPage)),
                            (lds_char*)(lds_void*)(dst + (2 * wave + p) * R::kPageBytes), source);
    }
  };
  // queries (B operand of S^T = K Q^T), zeros past the pairs
  uint4 qf[NS];
  {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + row;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)head * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = ld16(qp + (2 * s + half) * 8);
  }
  issue(KR{}, kpool, s_k, 0);
  issue(VR{}, vpool, s_v, 0);
  if (threadIdx.x == 0) s_bad = 0;                   // read and written behind the first unit's barriers
#pragma unroll
  for (int s = 0; s < NS; ++s) qf[s] = pair_ok ? qf[s] : make_uint4(0, 0, 0, 0);

  const lds_char* kbase = (const lds_char*)(lds_void*)s_k + 2 * wave * KR::kPageBytes + k_lane_base<RB, kFp8>(lane);
  const lds_char* vbase = (const lds_char*)(lds_void*)s_v + wave * VR::at(0, D * (int)sizeof(T) / 16 / kWaves) + v_lane_base<RB, kFp8>(lane);
  f32x16 o[NDW];
#pragma unroll
  for (int d = 0; d < NDW; ++d) o[d] = splat(0.0f);
  float m = -INFINITY, lsum = 0.0f;

  for (int u = 0; u < n_units; ++u) {
    const int key0 = k_begin + u * kUnitKeys;
    // ---- scores of this wave's block; its K has landed (V's loads may be in flight)
    __builtin_amdgcn_s_waitcnt(vm_wait(kLoads));
    asm volatile("" ::: "memory");
    f32x16 s = splat(0.0f);
#pragma unroll
    for (int ss = 0; ss < NS; ++ss) s = mfma32(widen(k_fragment<RB, kFp8>(kbase, ss)), qf[ss], s);
    __builtin_amdgcn_s_waitcnt(kLgkmWait);           // read: the buffer takes the next unit's
    asm volatile("" ::: "memory");
    issue(KR{}, kpool, s_k, u + 1);
    const int kb = key0 + 32 * wave;
    if (kb + 31 > first_n || kb < mask_lo) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kb + half * 4 + (r >> 2) * 8 + (r & 3);
        s[r] = (key <= row_n && key >= row_lo) ? s[r] : -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    const float2 mh = halves32(mx);
    s_mx[wave][lrow] = fmaxf(mh.x, mh.y) * a.scale_log2;      // both halves of the wave, the same value
    __syncthreads();
    // ---- the references of the unit's blocks in order (every wave alike), this wave's weights
    float alpha[kWaves], m_ref = 0.0f;
    bool raised[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      alpha[w] = raise_reference(m, s_mx[w][lrow], raised[w]);
      if (w == wave) m_ref = m == -INFINITY ? 0.0f : m;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -m_ref));
    float psum = 0.0f;
    s_p[wave][0][lane] = round_weights(s, 0, psum);
    s_p[wave][1][lane] = round_weights(s, 1, psum);
    const float2 ph = halves32(psum);
    s_sum[wave][lrow] = ph.x + ph.y;
    // V of the unit has landed (the next unit's K may be in flight)
    __builtin_amdgcn_s_waitcnt(vm_wait(kLoads));
    __syncthreads();
    // a masked key weighs 0, and 0 times an Inf or NaN would reach rows that do not see it (see the tile kernel)
    if (min(key0 + kUnitKeys, n_hi) - 1 > first_n || key0 < mask_lo) {
      if (finite_page<T, VR>(s_v + 2 * wave * VR::kPageBytes, lane) | finite_page<T, VR>(s_v + (2 * wave + 1) * VR::kPageBytes, lane)) s_bad = 1;
      __syncthreads();
    }
    // ---- this wave's dimensions over the unit's blocks
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      lsum = fmaf(lsum, alpha[w], s_sum[w][lrow]);
      if ((u > 0 || w > 0) && __builtin_amdgcn_ballot_w64(raised[w]) != 0) {      // O is 0 before the first block
#pragma unroll
        for (int d = 0; d < NDW; ++d) o[d] *= alpha[w];
      }
      const uint4 p0 = s_p[w][0][lane], p1 = s_p[w][1][lane];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < NDW; ++d)
          o[d] = mfma32(widen(v_fragment<RB, kFp8>(vbase + (2 * w + ks) * VR::kPageBytes, d)), ks ? p1 : p0, o[d]);
    }
    __syncthreads();                                 // V, weights and sums are read: the next unit's may come
    issue(VR{}, vpool, s_v, u + 1);
  }
  __builtin_amdgcn_s_waitcnt(vm_wait(0));            // the empty loads past the last unit write LDS: none may outlive the workgroup

  // ---- the segment's partial, or the result when there is one segment
  const int rank = a.part.n_seg > 1 ? few_rows_before(a, b) : 0;
  if (a.part.n_seg > 1 && rank + sq.len > a.few_rows) return;     // overlapping ranges hold more rows than there are
  auto slot_of = [&](int p) -> int64_t {
    const int h = g * a.group + (p & (a.group - 1));
    if (a.part.n_seg > 1) return (((int64_t)l * a.few_rows + rank + (p >> lg)) * a.Hq + h) * a.part.n_seg + seg;
    return ((int64_t)l * a.seqs.n_tokens + sq.row0 + (p >> lg)) * a.Hq + h;
  };
  if (pair_ok) {
    const int64_t at = slot_of(pair);
    if (a.part.n_seg > 1) {
      float* op = a.part.acc + at * D + wave * NDW * 32;
#pragma unroll
      for (int d = 0; d < NDW; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<float4*>(op + d * 32 + r4 * 8 + half * 4) =
              make_float4(o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]);
      if (wave == 0 && half == 0) *reinterpret_cast<float2*>(a.part.ml + at * 2) = make_float2(m, lsum);
    } else {
      const float inv = 1.0f / lsum;
      uint16_t* op = static_cast<uint16_t*>(a.out) + at * D + wave * NDW * 32;
#pragma unroll
      for (int d = 0; d < NDW; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<uint2*>(op + d * 32 + r4 * 8 + half * 4) =
              make_uint2(pack_bf16_rne(o[d][r4 * 4] * inv, o[d][r4 * 4 + 1] * inv),
                         pack_bf16_rne(o[d][r4 * 4 + 2] * inv, o[d][r4 * 4 + 3] * inv));
    }
  }
  if (s_bad != 0) {                                  // the values that are not finite, to the rows that see them
    __builtin_amdgcn_s_waitcnt(vm_wait(0));
    __syncthreads();
    if (wave != 0) return;
    put_bad_values(a, vpool, bt, g, k_begin, k_end, W, sq.ctx, lg, 0, n_pairs, [&](int p, int x, float v) {
      const int64_t at = slot_of(p) * D + x;
      if (a.part.n_seg > 1) {
        a.part.acc[at] = take_in(a.part.acc[at], v);
      } else {
        uint16_t* to = static_cast<uint16_t*>(a.out) + at;
        *to = (uint16_t)(__float_as_uint(take_in(bf16_bits_to_f32(*to), v)) >> 16);
      }
    });
  }
}

// The folds.  out = a row's segments folded in ascending order, in the operations of a tile kernel that walks all keys.
//
// Rows of the few kernel's: a lane a dimension of a (layer, row of the launch, query head).
template <int D>
__device__ __forceinline__ void fold_few(const PackedAttnArgs& a, const PackedPartials& part, uint32_t workgroup) {
  const int64_t id = (int64_t)workgroup * (256 / D) + __builtin_amdgcn_readfirstlane(threadIdx.x / D);
  const int x = threadIdx.x % D;
  const int h = (int)(id % a.Hq);
  const int t = (int)(id / a.Hq % a.few_rows), l = (int)(id / a.Hq / a.few_rows);
  if (l >= a.n_layers) return;
  const SeqUnit u = find_unit(a.seqs, t, [&](const SeqRange& s) { return is_few(a, s) ? s.len : 0; });
  if (u.b < 0) return;
  const int n = u.range.ctx + u.at;
  const int s_lo = window_start(layer_window(a, l), n + 1) / kPackedSeg, s_hi = n / kPackedSeg;
  const float* ml = part.ml + id * part.n_seg * 2;
  const float* acc = part.acc + id * part.n_seg * D + x;
  float m_run = -INFINITY, l_run = 0.0f, o_run = 0.0f;
#pragma unroll 8
  for (int s = s_lo; s <= s_hi; ++s) {
    const float2 y = *reinterpret_cast<const float2*>(ml + 2 * s);
    const FoldFactors f = fold_factors(m_run, l_run, y.x, y.y);
    o_run = fmaf(acc[(int64_t)s * D], f.part, o_run * f.run);
  }
  const int64_t row = (int64_t)l * a.seqs.n_tokens + u.range.row0 + u.at;
  static_cast<__bf16*>(a.out)[(row * a.Hq + h) * D + x] = (__bf16)(o_run * (1.0f / l_run));
}

// Tiles: a workgroup takes 32 dims of a block of 32 pairs, a wave 8 of them, a lane a pair and 4 dims.  Segments that the
// block's other rows see but the lane's row does not have weight 0 there.  T: type of the result.  kPairs: pairs of a tile.
template <typename T, int D, int kPairs>
__device__ __forceinline__ void fold_tiles(const PackedAttnArgs& a, const PackedPartials& part, uint32_t id) {
  constexpr int kBlocks = kPairs / 32, kAhead = 8;   // kAhead: segments requested at a time
  // (layer, tile, KV head, block, 32 dims)
  const int chunk = (int)(id % (D / 32)) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  id /= D / 32;
  const int i = (int)(id % kBlocks);
  id /= kBlocks;
  const int g = (int)(id % (uint32_t)a.Hkv);
  id /= (uint32_t)a.Hkv;
  const int slot = (int)(id % (uint32_t)a.n_tiles), l = (int)(id / (uint32_t)a.n_tiles);
  const int lg = 31 - __builtin_clz(a.group);
  const SeqUnit u = find_unit(a.seqs, slot, [&](const SeqRange& s) {
    return is_few(a, s) ? 0 : (int)((((int64_t)s.len << lg) + kPairs - 1) / kPairs);
  });
  if (u.b < 0) return;
  const int pair0 = (u.count - 1 - u.at) * kPairs + 32 * i;
  const int first = pair0 >> lg, last = min((pair0 + 31) >> lg, u.range.len - 1);
  if (first >= u.range.len) return;
  const int s_lo = window_start(layer_window(a, l), u.range.ctx + first + 1) / kPackedSeg, s_hi = (u.range.ctx + last) / kPackedSeg;
  const int lane = threadIdx.x & 63;
  const int64_t block = part_block(a, part.n_seg, l, slot, g, kBlocks, i, 0);
  const float* ml = part.ml + (block * 32 + (lane & 31)) * 2;
  const float* acc = part.acc + block * (32 * D) + (chunk * 64 + lane) * 4;
  float m_run = -INFINITY, l_run = 0.0f, o_run[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = s_lo; s0 <= s_hi; s0 += kAhead) {
    float2 x[kAhead];
    float4 v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int s = min(s0 + j, s_hi);
      x[j] = *reinterpret_cast<const float2*>(ml + s * 64);
      v[j] = *reinterpret_cast<const float4*>(acc + (int64_t)s * (32 * D));
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (s0 + j <= s_hi) {
        const FoldFactors f = fold_factors(m_run, l_run, x[j].x, x[j].y);
        o_run[0] = fmaf(v[j].x, f.part, o_run[0] * f.run);
        o_run[1] = fmaf(v[j].y, f.part, o_run[1] * f.run);
        o_run[2] = fmaf(v[j].z, f.part, o_run[2] * f.run);
        o_run[3] = fmaf(v[j].w, f.part, o_run[3] * f.run);
      }
  }
  const int p = pair0 + (lane & 31);
  if ((p >> lg) >= u.range.len) return;
  const int64_t row = ((int64_t)l * a.seqs.n_tokens + u.range.row0 + (p >> lg)) * a.Hq + g * a.group + (p & (a.group - 1));
  const float inv = 1.0f / l_run;
  struct alignas(4 * sizeof(T)) Four {
    T x[4];
  };
  *reinterpret_cast<Four*>(static_cast<T*>(a.out) + row * D + chunk * 8 + (lane >> 5) * 4) = {
      {(T)(o_run[0] * inv), (T)(o_run[1] * inv), (T)(o_run[2] * inv), (T)(o_run[3] * inv)}};
}

// Both in one launch: the few kernel's rows first, in few_workgroups workgroups (none beside fp32 caches, which it does not take).
template <typename T, int D, int kPairs>
__global__ __launch_bounds__(256) void packed_fold_kernel(const PackedAttnArgs a, const PackedPartials few, const uint32_t few_workgroups) {
  if constexpr (!std::is_same<T, float>::value) {
    if (blockIdx.x < few_workgroups) {
      fold_few<D>(a, few, blockIdx.x);
      return;
    }
  }
  fold_tiles<T, D, kPairs>(a, a.part, blockIdx.x - few_workgroups);
}

// Waves of a workgroup: four take a segment of a launch that leaves CUs idle soonest, two leave room for more
// workgroups on a CU, whose starts and ends then overlap.  Two against four, us, at workgroups (bf16 unless noted):
// head_dim 256: 80 27 / 20, 256 31 / 28, fp8 256 26 / 21, 512 45 / 53, 768 74 / 78, fp8 768 35 / 46, 4,224 (16 tokens over
// 33k keys) 521 / 650; 128: 128 23 / 18, 256 24 / 19, 512 27 / 25, 768 34 / 45, 8,448 528 / 577.
constexpr unsigned kFewGrid = 256;
template <typename T, int D>
void launch_few_d(const PackedAttnArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)packed_few_workgroups(a);
  constexpr int kMost = D == 64 ? 2 : 4;
  if (grid <= kFewGrid)
    packed_few_kernel<T, D, kMost><<<grid, 64 * kMost, 0, stream>>>(a);
  else
    packed_few_kernel<T, D, 2><<<grid, 64 * 2, 0, stream>>>(a);
}

template <typename T>
hipError_t launch_few_t(const PackedAttnArgs& a, hipStream_t stream) {
  switch (a.D) {
    case 64: launch_few_d<T, 64>(a, stream); break;
    case 128: launch_few_d<T, 128>(a, stream); break;
    case 256: launch_few_d<T, 256>(a, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T, int D, int kPairs>
hipError_t launch_fold_d(const PackedAttnArgs& a, const PackedPartials& few, hipStream_t stream) {
  const int64_t few_rows = few.n_seg > 1 ? (int64_t)a.n_layers * a.few_rows * a.Hq : 0;
  const unsigned few_workgroups = (unsigned)((few_rows + 256 / D - 1) / (256 / D));
  const unsigned tiles = a.part.n_seg > 1 ? (unsigned)packed_fold_workgroups(a, kPairs) : 0;
  packed_fold_kernel<T, D, kPairs><<<few_workgroups + tiles, 256, 0, stream>>>(a, few, few_workgroups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_few(const PackedAttnArgs& a, int dtype, hipStream_t stream) {
  if (dtype == kDtypeBf16) return launch_few_t<uint16_t>(a, stream);
  if (dtype == kDtypeFp8) return launch_few_t<uint8_t>(a, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_packed_fold(const PackedAttnArgs& a, const PackedPartials& few, int dtype, hipStream_t stream) {
  const bool f32 = dtype == kDtypeF32;
  switch (a.D) {
    case 64: return f32 ? launch_fold_d<float, 64, kF32Pairs>(a, few, stream) : launch_fold_d<__bf16, 64, kTilePairs>(a, few, stream);
    case 128: return f32 ? launch_fold_d<float, 128, kF32Pairs>(a, few, stream) : launch_fold_d<__bf16, 128, kTilePairs>(a, few, stream);
    case 256: return f32 ? launch_fold_d<float, 256, kF32Pairs>(a, few, stream) : launch_fold_d<__bf16, 256, kTilePairs>(a, few, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvg
