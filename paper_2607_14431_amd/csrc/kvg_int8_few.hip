// Attention over int8 caches of sequences with few rows (single tokens, short chunks): a workgroup per (layer, sequence, KV head,
// segment of kPackedSeg keys), up to kFewPairs (row, query head) pairs.  The fold of segments is packed_fold_kernel.
//
// The sums are those of the tile kernel (kvg_int8_tiles.hip), operation for operation, spread over the waves as in
// packed_few_kernel: the scores of a unit's blocks of 32 keys (a block per wave), then the weights, then the weighted values (a
// part of head_dim per wave, over all of the unit's blocks in order).
//
// Bound: many sequences, memory (16 tokens over 33k keys of 8 x 256: 306 us, 5.3 TB/s); one sequence, the chain of a workgroup: requests,
// their latency, scores, references, values (4.6k keys of 8 x 256: 24 us, 4 of them the fold; with a read of LDS between each two
// blocks, the query's loads under conditions and four waves it was 27).
#include "kvg_int8_mfma.h"
#include "kvg_launch.h"

namespace kvg {

namespace {

// s_waitcnt operand that waits for vmcnt <= n alone (gfx9 encoding: bits 3:0 and 15:14)
constexpr int vm_wait(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }
constexpr int kLgkmWait = 0xC07F;      // lgkmcnt(0) alone
constexpr int kStream = 2;             // buffer load policy: nontemporal (every row is read once; 16 tokens over 33k keys 306 us, plain 324)

// kWaves: waves of a workgroup, a block of 32 keys and D / kWaves dimensions each.  kDepth: units in LDS or on their way.
template <int D, int kWaves, int kDepth>
__global__ __launch_bounds__(64 * kWaves) void int8_few_kernel(const PackedAttnArgs a, const Int8Scales scales) {
  constexpr int NS = D / 32;
  constexpr int NDW = D / 32 / kWaves;               // 32-wide blocks of head_dim per wave
  constexpr int kUnitKeys = 32 * kWaves;
  using KR = KRows<D>;
  using VR = VRows<D>;
  constexpr int kLoads = 2 * KR::kPageLoads;         // direct loads of a wave's block, K or V
  static_assert(D / 32 % kWaves == 0 && kPackedSeg % kUnitKeys == 0, "units");
  constexpr int kKBytes = 2 * kWaves * KR::kPageBytes, kVBytes = 2 * kWaves * VR::kPageBytes;      // of a unit
  constexpr int kYounger = (2 * kDepth - 1) * kLoads;        // loads behind the ones that the next step reads
  static_assert(kYounger + kLoads < 64, "vmcnt");
  __shared__ __attribute__((aligned(1024))) char s_k[kDepth * kKBytes];
  __shared__ __attribute__((aligned(1024))) char s_v[kDepth * kVBytes];
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

  const int pair = min(lrow, n_pairs - 1);
  const bool pair_ok = lrow < n_pairs;
  const int row = pair >> lg, head = g * a.group + (pair & (a.group - 1));
  const int row_n = sq.ctx + row, row_lo = window_start(W, row_n + 1);

  const int64_t lbase = (int64_t)(a.layer0 + l) * a.layer_elems;
  const char* kpool = static_cast<const char*>(a.k_pool) + lbase;
  const char* vpool = static_cast<const char*>(a.v_pool) + lbase;

  // ---- the pages' scales and the query are requested first, and converted with the keys on their way
  const int64_t scale_at = ((int64_t)(a.layer0 + l) * a.n_pages + pg) * a.Hkv + g;
  const float scale_k = scales.k[scale_at], scale_v = scales.v[scale_at];
  uint4 raw[NS][2];
  {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + row;
    load_query<D>(raw, static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)head * D, half);
  }
  asm volatile("" ::: "memory");

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
  static_for<0, kDepth>([&](auto u) {
    issue(KR{}, kpool, s_k + decltype(u)::value * kKBytes, decltype(u)::value);
    issue(VR{}, vpool, s_v + decltype(u)::value * kVBytes, decltype(u)::value);
  });
  const PageScales page = page_scales(scale_k, scale_v);
  const uint32_t bad_pages = (uint32_t)__builtin_amdgcn_ballot_w64(page.bad);
  Int8Query<D> q;
  split_query<D>(q, raw);
  const float q_scale = q.step * a.scale_log2;

  const lds_char* kbase = (const lds_char*)(lds_void*)s_k + 2 * wave * KR::kPageBytes + k_lane_base<D, false>(lane);
  const lds_char* vbase = (const lds_char*)(lds_void*)s_v + wave * VR::at(0, D / 16 / kWaves) + v_lane_base<D, true>(lane);
  f32x16 o[NDW];
#pragma unroll
  for (int d = 0; d < NDW; ++d) o[d] = splat(0.0f);
  Int8State st = empty_state(q.finite ? 0.0f : kNaN);

  int slot = 0;                                      // u % kDepth
  for (int u = 0; u < n_units; ++u, slot = slot + 1 == kDepth ? 0 : slot + 1) {
    const int key0 = k_begin + u * kUnitKeys;
    // ---- scores of this wave's block; its K has landed (its V and later units may be in flight)
    __builtin_amdgcn_s_waitcnt(vm_wait(kYounger));
    asm volatile("" ::: "memory");
    i32x16 hi = (i32x16)(0), lo = (i32x16)(0);
#pragma unroll
    for (int ss = 0; ss < NS; ++ss) {
      const uint4 k = int8_k_fragment<D>(kbase + slot * kKBytes, ss);
      hi = mfma_i8(k, q.hi[ss], hi);
      lo = mfma_i8(k, q.lo[ss], lo);
    }
    __builtin_amdgcn_s_waitcnt(kLgkmWait);           // read: the buffer takes a later unit's
    asm volatile("" ::: "memory");
    issue(KR{}, kpool, s_k + slot * kKBytes, u + kDepth);
    const int kb = key0 + 32 * wave;
    auto lv_at = [&](int key) -> float { return lane_value(page.lv, (key / kPage) & 31); };
    float kq0 = key_factor(q_scale, lane_value(page.k, (kb / kPage) & 31));
    float kq1 = key_factor(q_scale, lane_value(page.k, (kb / kPage + 1) & 31));
    f32x16 s;
    float mx[2] = {-INFINITY, -INFINITY};
    const bool masked = kb + 31 > first_n || kb < mask_lo;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = (float)((hi[r] << 8) + lo[r]);
      if (masked) {
        const int key = kb + half * 4 + (r >> 2) * 8 + (r & 3);
        s[r] = (key <= row_n && key >= row_lo) ? s[r] : -INFINITY;
      }
      mx[r / 8] = fmaxf(mx[r / 8], s[r]);
    }
    {
      const float2 m = max_halves(mx[0], mx[1]);
      s_mx[wave][lrow] = make_float2(largest_score(m.x, kq0), largest_score(m.y, kq1));      // both halves of the wave, the same values
    }
    __syncthreads();
    // ---- the references of the unit's blocks in order (every wave alike), this wave's weights
    Int8Raise raise[kWaves];
    bool raised[kWaves];                             // seldom: the references are coarse
    Int8Page p0 = {}, p1 = {};
    float2 most[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most[w] = s_mx[w][lrow];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 x = most[w];
      const float lv0 = lv_at(key0 + 32 * w), lv1 = lv_at(key0 + 32 * w + kPage);
      const bool mine = is_raised(st, x.x, x.y, lv0, lv1);
      raised[w] = __builtin_amdgcn_ballot_w64(mine) != 0;
      if (raised[w]) raise[w] = raise_block(st, mine, x.x, x.y, lv0, lv1);
      if (w == wave) {
        p0 = page_weights(st, lv0);
        p1 = page_weights(st, lv1);
        if (__builtin_amdgcn_ballot_w64(is_far(st)) != 0) {
          far_page(s, 0, kq0, p0, st, lv0);
          far_page(s, 8, kq1, p1, st, lv1);
        }
      }
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = weight_of(s[r], r < 8 ? kq0 : kq1, r < 8 ? p0.c : p1.c);
      sum[r / 8] += s[r];
    }
    s_p[wave][0][lane] = round_weights8(s, 0);
    s_p[wave][1][lane] = round_weights8(s, 1);
    s_sum[wave][lrow] = block_sum(sum[0], sum[1], p0.back, p1.back);
    if (bad_pages != 0) {
      for (int i = 0; i < 2 * kWaves; ++i) {
        const int key = key0 + i * kPage;
        if ((bad_pages >> ((key / kPage) & 31) & 1) != 0 && key <= row_n && key + kPage > row_lo) st.l = kNaN;
      }
    }
    // V of the unit has landed (later units may be in flight)
    __builtin_amdgcn_s_waitcnt(vm_wait(kYounger));
    __syncthreads();
    // ---- this wave's dimensions over the unit's blocks: all reads first
    uint2 v[kWaves][2][NDW];
    uint4 p[kWaves][2];
    float sums[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      sums[w] = s_sum[w][lrow];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        p[w][ks] = s_p[w][ks][lane];
#pragma unroll
        for (int d = 0; d < NDW; ++d) v[w][ks][d] = v_fragment<D, true>(vbase + slot * kVBytes + (2 * w + ks) * VR::kPageBytes, d);
      }
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (raised[w]) {
        st.l *= raise[w].alpha_l;
        if (u > 0 || w > 0) {                        // O is 0 before the first block
#pragma unroll
          for (int d = 0; d < NDW; ++d) o[d] *= raise[w].alpha_o;
        }
      }
      st.l += sums[w];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int d = 0; d < NDW; ++d) o[d] = mfma_f16(widen_int8(v[w][ks][d]), p[w][ks], o[d]);
    }
    __syncthreads();                                 // V, weights and sums are read: a later unit's may come
    issue(VR{}, vpool, s_v + slot * kVBytes, u + kDepth);
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
            make_uint2(pack_bf16_rne(row_result(o[d][r4 * 4], inv), row_result(o[d][r4 * 4 + 1], inv)),
                       pack_bf16_rne(row_result(o[d][r4 * 4 + 2], inv), row_result(o[d][r4 * 4 + 3], inv)));
  }
}

// Up to this many workgroups, one a compute unit, a workgroup has waves for all of head_dim and, where LDS holds them, all keys of a
// segment on their way at once: the time is one workgroup's, start to end.  More workgroups hide their waits from each other: two
// waves each and one unit (16 tokens over 33k keys of head_dim 256: 306 us, with four waves 354).  Small workgroups against
// large ones, each with the fold, us, at workgroups: head_dim 256: 80 30 / 25, 160 33 / 26, 240 33 / 27, 320 38 / 43, 1,280 53 / 84; 128: 16
// 17 / 15, 80 26 / 21, 160 25-26 / 20-22, 320 28-30 / 27, 640 30-32 / 42-49, 1,280 35 / 63.  At head_dim 64 it is the same kernel (a deep one of 8 units: 48 20.0 / 20.4, 576 26 / 28).
constexpr unsigned kFewGrid = 256;
template <int D>
hipError_t launch_few_d(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream) {
  const unsigned grid = (unsigned)packed_few_workgroups(a);
  constexpr int kMost = D / 32, kDeep = D == 128 ? 4 : 1;
  if (grid <= kFewGrid)
    int8_few_kernel<D, kMost, kDeep><<<grid, 64 * kMost, 0, stream>>>(a, s);
  else
    int8_few_kernel<D, 2, 1><<<grid, 64 * 2, 0, stream>>>(a, s);
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
