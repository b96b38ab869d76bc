// Attention over int8 caches of sequences with few rows (single tokens, short chunks): a workgroup per (layer, sequence, KV head,
// segment of kPackedSeg keys), up to kFewPairs (row, query head) pairs.  The fold of segments is packed_fold_kernel.
//
// The sums are those of the tile kernel (kvg_int8_tiles.hip), operation for operation, spread over the waves as in
// packed_few_kernel: the scores of a unit's blocks of 32 keys (a block per wave), then the weights, then the weighted values (a
// part of head_dim per wave, over all of the unit's blocks in order).
#include "kvg_int8_mfma.h"
#include "kvg_launch.h"

namespace kvg {

namespace {

// s_waitcnt operand that waits for vmcnt <= n alone (gfx9 encoding: bits 3:0 and 15:14)
constexpr int vm_wait(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }
constexpr int kLgkmWait = 0xC07F;      // lgkmcnt(0) alone
constexpr int kStream = 2;             // buffer load policy: nontemporal (every row is read once)

// kWaves: waves of a workgroup, a block of 32 keys and D / kWaves dimensions each
template <int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void int8_few_kernel(const PackedAttnArgs a, const Int8Scales scales) {
  constexpr int NS = D / 32;
  constexpr int NDW = D / 32 / kWaves;               // 32-wide blocks of head_dim per wave
  constexpr int kUnitKeys = 32 * kWaves;
  using KR = KRows<D>;
  using VR = VRows<D>;
  constexpr int kLoads = 2 * KR::kPageLoads;         // direct loads of a wave's block, K or V
  static_assert(D / 32 % kWaves == 0 && kPackedSeg % kUnitKeys == 0, "units");
  __shared__ __attribute__((aligned(1024))) char s_k[2 * kWaves * KR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char s_v[2 * kWaves * VR::kPageBytes];
  __shared__ uint4 s_p[kWaves][2][64];
  __shared__ float2 s_mx[kWaves][32];
  __shared__ float s_sum[kWaves][32];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lrow = lane & 31, half = lane >> 5;
  const int lg = 31 - __builtin_clz(a.group);
  // (layer, sequence, segment, KV head), the KV head fastest: workgroups without work come in runs
  uint32_t id = blockIdx.x;
  const int g = (int)(id % (uint32_t)a.Hkv);
  id /= (uint32_t)a.Hkv;
  int seg = (int)(id % (uint32_t)a.part.n_seg);
  id /= (uint32_t)a.part.n_seg;
  const int b = (int)(id % (uint32_t)a.seqs.batch);
  const int l = (int)(id / (uint32_t)a.seqs.batch);
  seg = (int)((uint32_t)(seg + b) % (uint32_t)a.part.n_seg);
  const int32_t* bt = a.seqs.tables + (int64_t)b * a.seqs.max_pages;
  // page ids of the segment, one per lane (requested with the sequence's range), and their scales
  int32_t pg = bt[min(seg * (kPackedSeg / kPage) + (lane & 31), a.seqs.max_pages - 1)];
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
  pg = pg >= 0 && pg < a.n_pages ? pg : 0;
  const int64_t scale_at = ((int64_t)(a.layer0 + l) * a.n_pages + pg) * a.Hkv + g;
  const float k_scale = scales.k[scale_at], v_scale = scales.v[scale_at];

  const int pair = min(lrow, n_pairs - 1);
  const bool pair_ok = lrow < n_pairs;
  const int row = pair >> lg, head = g * a.group + (pair & (a.group - 1));
  const int row_n = sq.ctx + row, row_lo = window_start(W, row_n + 1);

  const int64_t lbase = (int64_t)(a.layer0 + l) * a.layer_elems;
  const char* kpool = static_cast<const char*>(a.k_pool) + lbase;
  const char* vpool = static_cast<const char*>(a.v_pool) + lbase;

  // ---- loads of this wave's block of unit u (two pages, K or V); rows from k_end on read as zeros
  const int source = KR::source(lane);               // the same for V
  auto issue = [&](auto rows_type, const char* pool, char* dst, int u) {
    using R = decltype(rows_type);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int key = k_begin + u * kUnitKeys + wave * 32 + p * kPage;
      const int32_t page = __builtin_amdgcn_readlane(pg, (key / kPage) & 31);
      load_page<R, kStream>(pool + ((int64_t)page * a.Hkv + g) * kPage * D, __builtin_amdgcn_readfirstlane(min(max(k_end - key, 0), kPage)),
                            (lds_char*)(lds_void*)(dst + (2 * wave + p) * R::kPageBytes), source);
    }
  };
  auto scales_at = [&](int key) -> PageScales {      // of the page that holds it
    const int p = (key / kPage) & 31;
    return page_scales(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), p)),
                       __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scale), p)));
  };
  issue(KR{}, kpool, s_k, 0);
  issue(VR{}, vpool, s_v, 0);
  Int8Query<D> q;
  {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + row;
    load_query<D>(q, static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)head * D, pair_ok, half);
  }
  const float q_scale = q.step * a.scale_log2;

  const lds_char* kbase = (const lds_char*)(lds_void*)s_k + 2 * wave * KR::kPageBytes + k_lane_base<D, false>(lane);
  const lds_char* vbase = (const lds_char*)(lds_void*)s_v + wave * VR::at(0, D / 16 / kWaves) + v_lane_base<D, true>(lane);
  f32x16 o[NDW];
#pragma unroll
  for (int d = 0; d < NDW; ++d) o[d] = splat(0.0f);
  Int8State st = {-INFINITY, -INFINITY, 0.0f};

  __builtin_amdgcn_s_waitcnt(vm_wait(0));            // the first unit, with the query requested behind it
  for (int u = 0; u < n_units; ++u) {
    const int key0 = k_begin + u * kUnitKeys;
    // ---- scores of this wave's block; its K has landed (V's loads may be in flight)
    __builtin_amdgcn_s_waitcnt(vm_wait(kLoads));
    asm volatile("" ::: "memory");
    i32x16 hi = (i32x16)(0), lo = (i32x16)(0);
#pragma unroll
    for (int ss = 0; ss < NS; ++ss) {
      const uint4 k = int8_k_fragment<D>(kbase, ss);
      hi = mfma_i8(k, q.hi[ss], hi);
      lo = mfma_i8(k, q.lo[ss], lo);
    }
    __builtin_amdgcn_s_waitcnt(kLgkmWait);           // read: the buffer takes the next unit's
    asm volatile("" ::: "memory");
    issue(KR{}, kpool, s_k, u + 1);
    const int kb = key0 + 32 * wave;
    const PageScales own0 = scales_at(kb), own1 = scales_at(kb + kPage);
    f32x16 s = int8_scores(hi, lo, q_scale * own0.k, q_scale * own1.k);
    if (kb + 31 > first_n || kb < mask_lo) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kb + half * 4 + (r >> 2) * 8 + (r & 3);
        s[r] = (key <= row_n && key >= row_lo) ? s[r] : -INFINITY;
      }
    }
    s_mx[wave][lrow] = page_maxima(s);               // both halves of the wave, the same values
    __syncthreads();
    // ---- the references of the unit's blocks in order (every wave alike), this wave's weights
    float alpha_l[kWaves], alpha_o[kWaves];
    bool raised[kWaves];
    Int8Block mine = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 x = s_mx[w][lrow];
      const Int8Block blk = raise_block(st, x.x, x.y, scales_at(key0 + 32 * w), scales_at(key0 + 32 * w + kPage));
      alpha_l[w] = blk.alpha_l;
      alpha_o[w] = blk.alpha_o;
      raised[w] = blk.raised;
      if (w == wave) mine = blk;
    }
    uint4 p[2];
    s_sum[wave][lrow] = block_weights(s, mine, p);
    s_p[wave][0][lane] = p[0];
    s_p[wave][1][lane] = p[1];
    // V of the unit has landed (the next unit's K may be in flight)
    __builtin_amdgcn_s_waitcnt(vm_wait(kLoads));
    __syncthreads();
    // ---- this wave's dimensions over the unit's blocks
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      st.l = fmaf(st.l, alpha_l[w], s_sum[w][lrow]);
      if ((u > 0 || w > 0) && __builtin_amdgcn_ballot_w64(raised[w]) != 0) {      // O is 0 before the first block
#pragma unroll
        for (int d = 0; d < NDW; ++d) o[d] *= alpha_o[w];
      }
      const uint4 p0 = s_p[w][0][lane], p1 = s_p[w][1][lane];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < NDW; ++d)
          o[d] = mfma_f16(widen_int8(v_fragment<D, true>(vbase + (2 * w + ks) * VR::kPageBytes, d)), ks ? p1 : p0, o[d]);
    }
    __syncthreads();                                 // V, weights and sums are read: the next unit's may come
    issue(VR{}, vpool, s_v, u + 1);
  }
  __builtin_amdgcn_s_waitcnt(vm_wait(0));            // the empty loads past the last unit write LDS: none may outlive the workgroup
  const int e = end_exponent(st);
#pragma unroll
  for (int d = 0; d < NDW; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = __builtin_ldexpf(o[d][r], e);

  // ---- the segment's partial, or the result when there is one segment
  const int rank = a.part.n_seg > 1 ? few_rows_before(a, b) : 0;
  if (a.part.n_seg > 1 && rank + sq.len > a.few_rows) return;     // overlapping ranges hold more rows than there are
  if (!pair_ok) return;
  if (a.part.n_seg > 1) {
    const int64_t at = (((int64_t)l * a.few_rows + rank + row) * a.Hq + head) * a.part.n_seg + seg;
    float* op = a.part.acc + at * D + wave * NDW * 32;
#pragma unroll
    for (int d = 0; d < NDW; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<float4*>(op + d * 32 + r4 * 8 + half * 4) =
            make_float4(o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]);
    if (wave == 0 && half == 0) *reinterpret_cast<float2*>(a.part.ml + at * 2) = make_float2(st.m, st.l);
  } else {
    const int64_t at = ((int64_t)l * a.seqs.n_tokens + sq.row0 + row) * a.Hq + head;
    const float inv = 1.0f / st.l;
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

constexpr unsigned kFewGrid = 256;
template <int D>
hipError_t launch_few_d(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream) {
  const unsigned grid = (unsigned)packed_few_workgroups(a);
  constexpr int kMost = D == 64 ? 2 : 4;
  if (grid <= kFewGrid)
    int8_few_kernel<D, kMost><<<grid, 64 * kMost, 0, stream>>>(a, s);
  else
    int8_few_kernel<D, 2><<<grid, 64 * 2, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_int8_few(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_few_d<64>(a, s, stream);
    case 128: return launch_few_d<128>(a, s, stream);
    case 256: return launch_few_d<256>(a, s, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvg
