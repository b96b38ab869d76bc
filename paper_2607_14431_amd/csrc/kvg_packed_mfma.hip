// Causal attention of packed sequences over a paged bf16 or fp8 cache, on bf16 MFMA (v_mfma_f32_32x32x16_bf16).
//
// Workgroup = (layer, KV head g, tile of a sequence): BM (row, query head) pairs of the sequence, heads
// fastest, 32 per wave.  Keys come in tiles of 64 (absolute multiples of 64 of the
// logical index) in two LDS stages, loaded with buffer_load ... lds while the tile before is computed.
//
// A row's sums have one order, whatever the launch: keys in blocks of 32, an online softmax over the blocks of a
// segment of kPackedSeg keys (absolute multiples), and the segments' states folded in ascending order.  A
// workgroup that walks all keys folds in registers; split launches leave one partial per segment for
// packed_fold_kernel (kvg_packed_few.hip), which folds them with the same operations.  Sequences of at most kFewPairs
// pairs are left to packed_few_kernel, which takes the same operations too.
//
//   S^T = K Q^T    A = K rows from LDS, B = the pairs' queries in registers; a lane owns one pair (lane % 32) and 16
//                  of a block's 32 keys, the other 16 are in lane ^ 32
//   softmax        fp32; the reference is the largest score rounded up to a multiple of kStep in log2 units and moves
//                  only when a block exceeds it, so states of different segments mostly share it and
//                  fold by one addition; weights are rounded to bf16 and summed as rounded, so a row of one key
//                  gives its value exactly and rounding errors of the heavy weights cancel
//   O^T += V^T P^T A = V^T fragments (ds_read_b64_tr), B = P straight from the S^T registers
//
// What bounds it: the matrix cores and the LDS together.  A fragment of 1 KiB takes the LDS 8 cycles and feeds one matrix
// step of 32, and four waves read at a time: both are busy alike, with the softmax's vector work (at head_dim 128 as many
// cycles again) and the waits between them.  A prompt of 12,288 tokens (16 / 8 heads x 256, bf16) takes 1,242 us: 1.00 PFLOP/s,
// matrix cores 48% busy; eight of up to 4,096 (32 / 16 x 128) 480 us: 0.81 PFLOP/s, 37% (medians of 200 calls in a row; the
// first ones of a run take up to a sixth longer, and cards differ by as much as 8%).  Two blocks of 32 pairs a wave, which halve the
// fragments, were slower when tried: 1.25 times at head_dim 128 (one wave a SIMD then), 1.4 times at 64.
#include "kvg_launch.h"
#include "kvg_packed_mfma.h"

#include <math.h>

#include <type_traits>

namespace kvg {

namespace {

constexpr int kTileKeys = 64;
constexpr int kSegTiles = kPackedSeg / kTileKeys;
constexpr int kWaves = 4;
// T: cache storage (uint16_t bf16, uint8_t fp8 E4M3).  kSplitKeys: a workgroup takes one segment and leaves its partial.
template <typename T, int D, bool kSplitKeys>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void packed_tiles_kernel(const PackedAttnArgs a) {
  constexpr bool kFp8 = sizeof(T) == 1;
  constexpr int RB = D * (int)sizeof(T);   // bytes per cache row
  constexpr int NS = D / 16;               // MFMA steps over head_dim
  constexpr int ND = D / 32;               // 32-wide blocks of head_dim
  constexpr int BM = kTilePairs;
  static_assert(BM == 32 * kWaves, "a block of 32 pairs per wave");
  // Fragments ahead of their use at D <= 128: a row block's worth where the registers hold it (the others: prompts of up
  // to 4,096 tokens, 32 / 16 heads x 128: four, five or six 465 to 478 us, with seven registers spilled each; eight 764).
  constexpr int kRing = kSplitKeys || D == 64 ? NS : 6;
  // A tile's loads among the matrix steps, or all at its start: 12,288 tokens at head_dim 256 1,158 us / 1,310 (fp8 1,244 /
  // 1,303); those prompts at 128 464 to 476 / 466, at 64 273 / 274 (fp8 280 / 271).
  constexpr bool kSpread = D != 128;
  using KR = KRows<RB>;
  using VR = VRows<RB>;
  // a wave brings one page of a tile; the V stages first, where an LDS instruction's immediate offset reaches
  __shared__ __attribute__((aligned(1024))) char sA_V0[kWaves * VR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char sA_V1[kWaves * VR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char sB_K0[kWaves * KR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char sB_K1[kWaves * KR::kPageBytes];
  __shared__ int s_bad;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int lrow = lane & 31, half = lane >> 5;
  const int lg = 31 - __builtin_clz(a.group);            // 1, 2, 4 or 8 query heads per KV head

  // ---- (tile, layer, segment, KV head), the KV head fastest (an XCD's workgroups share few heads); late tiles, which have
  // the most keys, first.  Workgroups without work come in runs: an XCD's go to its four shader engines in turn, and with
  // the tile before the segment one in four had work, all on the same engine: 35 rows over 32k keys (fp8), 69 -> 205 us.
  uint32_t id = blockIdx.x;
  const int g = (int)(id % (uint32_t)a.Hkv);
  id /= (uint32_t)a.Hkv;
  int seg = 0;
  if constexpr (kSplitKeys) {
    seg = (int)(id % (uint32_t)a.part.n_seg);
    id /= (uint32_t)a.part.n_seg;
  }
  const int l = (int)(id % (uint32_t)a.n_layers);
  const int slot = (int)(id / (uint32_t)a.n_layers);
  if constexpr (kSplitKeys) seg = (int)((uint32_t)(seg + slot) % (uint32_t)a.part.n_seg);      // a segment not always on the same XCD
  const SeqUnit u = find_unit(a.seqs, slot, [&](const SeqRange& s) {
    return is_few(a, s) ? 0 : (int)((((int64_t)s.len << lg) + BM - 1) / BM);
  });
  if (u.b < 0) return;
  const SeqRange sq = u.range;
  const int tile_id = u.count - 1 - u.at;
  const int ctx = sq.ctx, len = sq.len;

  const int pair0 = tile_id * BM + wave * 32;   // this wave's first pair
  const int W = layer_window(a, l);
  const int row = (pair0 + lrow) >> lg;
  const bool row_ok = row < len;
  const int row_n = ctx + row, row_lo = window_start(W, row_n + 1);      // this lane's row's visible keys [row_lo, row_n]
  const int first_row = pair0 >> lg;
  const int last_row = min((pair0 + 31) >> lg, len - 1);
  const bool idle = first_row >= len;                       // a wave without rows
  const int wave_first = ctx + first_row, wave_last = idle ? -1 : ctx + last_row;
  const int tile_first = ctx + ((tile_id * BM) >> lg);       // the workgroup's first row, and the first key all of its rows see
  const int tile_mask_lo = window_start(W, ctx + min((((tile_id + 1) * BM - 1) >> lg), len - 1) + 1);
  const int wave_lo = window_start(W, wave_first + 1), mask_lo = window_start(W, ctx + last_row + 1);
  const int n_hi = ctx + min(((tile_id + 1) * BM + a.group - 1) >> lg, len);   // keys [0, n_hi) needed by the workgroup
  int kt_begin = window_start(W, ctx + ((tile_id * BM) >> lg) + 1) / kTileKeys;
  int n_tiles = (n_hi + kTileKeys - 1) / kTileKeys;
  if constexpr (kSplitKeys) {
    kt_begin = max(kt_begin, seg * kSegTiles);
    n_tiles = min(n_tiles, (seg + 1) * kSegTiles);
    if (kt_begin >= n_tiles) return;
  }
  const int last_page = (n_hi - 1) / kPage;
  const int32_t* bt = a.seqs.tables + (int64_t)u.b * a.seqs.max_pages;
  const int64_t lbase = (int64_t)(a.layer0 + l) * a.layer_elems;
  const T* kpool = reinterpret_cast<const T*>(a.k_pool) + lbase;
  const T* vpool = reinterpret_cast<const T*>(a.v_pool) + lbase;

  // ---- loads: wave w brings page w of tile kt; rows past the last one the workgroup needs read as zeros
  const int source = KR::source(lane);     // the same for V
  auto page_slot = [&](int kt) { return kt * (kTileKeys / kPage) + wave; };
  auto page_of_tile = [&](int kt) -> int32_t { return bt[min(page_slot(kt), last_page)]; };
  struct PageSource {
    int64_t off;
    int rows;
  };
  auto tile_source = [&](int kt, int32_t page) -> PageSource {
    page = __builtin_amdgcn_readfirstlane(page);
    page = (page >= 0 && page < a.n_pages) ? page : 0;
    return {((int64_t)page * a.Hkv + g) * kPage * D, __builtin_amdgcn_readfirstlane(min(max(n_hi - page_slot(kt) * kPage, 0), kPage))};
  };
  constexpr int kTileLoads = 2 * KR::kPageLoads;       // of a wave: K and V alternate
  auto issue = [&](const PageSource& src, auto dst_stage, int j0, int j1) {
    constexpr int DS = decltype(dst_stage)::value;
    lds_char* dk = (lds_char*)(lds_void*)((DS ? sB_K1 : sB_K0) + wave * KR::kPageBytes);
    lds_char* dv = (lds_char*)(lds_void*)((DS ? sA_V1 : sA_V0) + wave * VR::kPageBytes);
    load_page<KR, 0>(kpool + src.off, src.rows, dk, source, (j0 + 1) / 2, (j1 + 1) / 2);
    load_page<VR, 0>(vpool + src.off, src.rows, dv, source, j0 / 2, j1 / 2);
  };

  // ---- queries (B operand of S^T), zeros past the rows
  uint4 qf[NS];
  {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (row_ok ? row : 0);
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)(g * a.group + ((pair0 + lrow) & (a.group - 1))) * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = row_ok ? ld16(qp + (2 * s + half) * 8) : make_uint4(0, 0, 0, 0);
  }

  f32x16 o[ND], o_run[kSplitKeys ? 1 : ND];
  float m = -INFINITY, lsum = 0.0f, m_run = -INFINITY, l_run = 0.0f;
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    o[d] = splat(0.0f);
    if constexpr (!kSplitKeys) o_run[d] = splat(0.0f);
  }

  const int k_lane = k_lane_base<RB, kFp8>(lane), v_lane = v_lane_base<RB, kFp8>(lane);

  if (tid == 0) s_bad = 0;              // read and written behind the first tile's barrier
  using Stage0 = std::integral_constant<int, 0>;
  using Stage1 = std::integral_constant<int, 1>;
  int32_t pg_next = page_of_tile(kt_begin);
  issue(tile_source(kt_begin, pg_next), Stage0{}, 0, kTileLoads);
  pg_next = page_of_tile(kt_begin + 1);

  bool fresh = true;                      // no block of the segment yet
  auto tile = [&](auto stage, int kt) __attribute__((always_inline)) {
    constexpr int ST = decltype(stage)::value;
    using Next = std::integral_constant<int, 1 - ST>;
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's share of tile kt (and the next page id) is here
    __syncthreads();                      // all of tile kt is in LDS; the other stage is no longer read
    const int key0 = kt * kTileKeys;
    // A masked key weighs 0, and 0 times an Inf or NaN among its values would reach rows that do not see it.  In tiles with
    // keys that some row of the workgroup does not see (the diagonal's, a window's lower edge; keys past n_hi
    // are zeros) such values are set to 0, and the rows that see them are given them at the end.
    if (min(key0 + kTileKeys, n_hi) - 1 > tile_first || key0 < tile_mask_lo) {
      if (finite_page<T, VR>((ST ? sA_V1 : sA_V0) + wave * VR::kPageBytes, lane)) s_bad = 1;
      __syncthreads();
    }
    const PageSource next = tile_source(kt + 1, pg_next);
    pg_next = page_of_tile(kt + 2);
    const bool unseen = key0 > wave_last || key0 + kTileKeys <= wave_lo;       // by this wave's rows
    if (!kSpread || unseen) issue(next, Next{}, 0, kTileLoads);
    if (unseen) return;
    // loads of step t (0 <= t < 2 NS over phases A and B)
    auto issue_step = [&](int t) {
      if constexpr (!kSpread) return;
      issue(next, Next{}, t * kTileLoads / (2 * NS), (t + 1) * kTileLoads / (2 * NS));
    };
    const lds_char* kbase = (const lds_char*)(lds_void*)(ST ? sB_K1 : sB_K0) + k_lane;
    const lds_char* vbase = (const lds_char*)(lds_void*)(ST ? sA_V1 : sA_V0) + v_lane;
    auto kread = [&](int f) { return k_fragment<RB, kFp8>(kbase + KR::at(32 * (f / NS), 0), f % NS); };        // f = block * NS + step
    auto vread = [&](int t) { return v_fragment<RB, kFp8>(vbase + VR::at(16 * (t / ND), 0), t % ND); };        // t = 16-key step * ND + d

    f32x16 s[2];
    if constexpr (D > 128) s[0] = s[1] = splat(0.0f);
    const bool need_mask = key0 + kTileKeys - 1 > wave_first || key0 < mask_lo;
    auto mask_block = [&](int kb) {
      if (need_mask) {
        const int at = D <= 128 ? 0 : kb;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // key - row_lo as unsigned: keys below the window wrap round
          const uint32_t key = key0 + kb * 32 + half * 4 - row_lo + (r >> 2) * 8 + (r & 3);
          s[at][r] = key <= (uint32_t)(row_n - row_lo) ? s[at][r] : -INFINITY;
        }
      }
    };
    // softmax of one block in 16 pieces, to sit beside the matrix steps of another phase: 0-3 the largest
    // score, 4 the reference, 5-12 two exponentials each, 13-14 rounding of eight weights and their sum, 15 the sum
    uint4 pf[2][2];
    struct {
      float mx, alpha, m_ref, psum;
      bool raised;
    } x;
    auto soft_piece = [&](int kb, int j) {
      if (j < 4) {
        if (j == 0) x.mx = -INFINITY;
#pragma unroll
        for (int r = 4 * j; r < 4 * j + 4; ++r) x.mx = fmaxf(x.mx, s[kb][r]);
      } else if (j == 4) {
        const float2 mh = halves32(x.mx);
        x.alpha = raise_reference(m, fmaxf(mh.x, mh.y) * a.scale_log2, x.raised);
        x.m_ref = m == -INFINITY ? 0.0f : m;      // no key seen yet: every weight is 0
        x.psum = 0.0f;
      } else if (j < 13) {
#pragma unroll
        for (int r = 2 * (j - 5); r < 2 * (j - 5) + 2; ++r)
          s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale_log2, -x.m_ref));
      } else if (j < 15) {
        pf[kb][j - 13] = round_weights(s[kb], j - 13, x.psum);
      } else {
        const float2 ph = halves32(x.psum);
        lsum = fmaf(lsum, x.alpha, ph.x + ph.y);
      }
    };
    // O of a segment's first block is still 0
    auto rescale_o = [&]() {
      if (!fresh && __builtin_amdgcn_ballot_w64(x.raised) != 0) {
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= x.alpha;
      }
      fresh = false;
    };
    // K fragments of both blocks form one stream read LK ahead of their MFMAs, V^T fragments one read LV ahead, whose first
    // LV are issued with block 1's scores (four, six or eight ahead: 12,288 tokens 1,252 to 1,258 us, fp8 1,313 to 1,319; fp8
    // fragments widened beside their reads, when tried, a fifth more)
    if constexpr (D <= 128) {
      // Two waves a SIMD: one's softmax runs beside the other's matrix steps.  The tile's K and V^T fragments, in the order of
      // their use, pass through one ring: a fragment's place is refilled with the one LR steps on.
      static_assert(NS == 2 * ND, "as many K as V^T fragments a block");
      constexpr int LR = kRing;
      Fragment<kFp8> ring[LR];
      auto fetch = [&](int t) {
        if (t < 4 * NS) ring[t % LR] = (t / NS) % 2 == 0 ? kread(t / (2 * NS) * NS + t % NS) : vread(t / (2 * NS) * NS + t % NS);
      };
#pragma unroll
      for (int t = 0; t < LR; ++t) fetch(t);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int ss = 0; ss < NS; ++ss) {
          const int t = 2 * kb * NS + ss;
          s[0] = mfma32(widen(ring[t % LR]), qf[ss], ss ? s[0] : splat(0.0f));
          fetch(t + LR);
          issue_step(kb * NS + ss);
          __builtin_amdgcn_sched_barrier(0);
        }
        mask_block(kb);
#pragma unroll
        for (int j = 0; j < 16; ++j) soft_piece(0, j);
        rescale_o();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const int t = (2 * kb + 1) * NS + i;
          o[i % ND] = mfma32(widen(ring[t % LR]), pf[0][i / ND], o[i % ND]);
          fetch(t + LR);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      return;
    }
    constexpr int LK = kFp8 ? 8 : 4;
    constexpr int RK = LK + 1;
    constexpr int NT = 4 * ND;
    constexpr int LV = kFp8 ? 8 : 4;
    constexpr int RV = LV + 1;
    Fragment<kFp8> kf[RK], vf[RV];
    auto kfetch = [&](int f) {
      if (f < 2 * NS) kf[f % RK] = kread(f);
    };
    auto vfetch = [&](int t) {
      if (t < NT) vf[t % RV] = vread(t);
    };
#pragma unroll
    for (int f = 0; f < LK; ++f) kfetch(f);
    // phase A: scores of block 0
#pragma unroll
    for (int ss = 0; ss < NS; ++ss) {
      kfetch(ss + LK);
      issue_step(ss);
      __builtin_amdgcn_sched_barrier(0);
      s[0] = mfma32(widen(kf[ss % RK]), qf[ss], s[0]);
      __builtin_amdgcn_sched_barrier(0);
    }
    mask_block(0);
    // phase B: scores of block 1 beside the softmax of block 0
    constexpr int kPieces = 16;
    static_assert(D <= 128 || LV <= NS, "first V^T fragments");
#pragma unroll
    for (int ss = 0; ss < NS; ++ss) {
      const int f = NS + ss;
      kfetch(f + LK);
      issue_step(NS + ss);
      if (ss >= NS - LV) vfetch(ss - (NS - LV));
      s[1] = mfma32(widen(kf[f % RK]), qf[ss], s[1]);
#pragma unroll
      for (int j = ss * kPieces / NS; j < (ss + 1) * kPieces / NS; ++j) soft_piece(0, j);
      __builtin_amdgcn_sched_barrier(0);
    }
    rescale_o();
    mask_block(1);
    // phases C and D: O^T += V^T P^T over block 0, beside the softmax of block 1, and over block 1
#pragma unroll
    for (int t = 0; t < 2 * ND; ++t) {
      vfetch(t + LV);
      o[t % ND] = mfma32(widen(vf[t % RV]), pf[0][t / ND], o[t % ND]);
#pragma unroll
      for (int j = t * kPieces / (2 * ND); j < (t + 1) * kPieces / (2 * ND); ++j) soft_piece(1, j);
      __builtin_amdgcn_sched_barrier(0);
    }
    rescale_o();
#pragma unroll
    for (int t = 2 * ND; t < NT; ++t) {
      vfetch(t + LV);
      __builtin_amdgcn_sched_barrier(0);
      o[t % ND] = mfma32(widen(vf[t % RV]), pf[1][t / ND - 2], o[t % ND]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // end of a segment: its state folded into the running one, which packed_fold_kernel does with the same operations
  auto fold = [&]() {
    if constexpr (!kSplitKeys) {
      const FoldFactors f = fold_factors(m_run, l_run, m, lsum);
      if (__builtin_amdgcn_ballot_w64(f.run != 1.0f || f.part != 1.0f) == 0) {
#pragma unroll
        for (int d = 0; d < ND; ++d) o_run[d] += o[d];
      } else {
#pragma unroll
        for (int d = 0; d < ND; ++d) o_run[d] = __builtin_elementwise_fma(o[d], splat(f.part), o_run[d] * f.run);
      }
      m = -INFINITY;
      lsum = 0.0f;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = splat(0.0f);
      fresh = true;
    }
  };
  auto step = [&](auto stage, int kt) __attribute__((always_inline)) {
    tile(stage, kt);
    if (!kSplitKeys && (kt + 1) % kSegTiles == 0 && kt + 1 < n_tiles) fold();
  };
  for (int kt = kt_begin; kt < n_tiles; kt += 2) {
    step(Stage0{}, kt);
    if (kt + 1 < n_tiles) step(Stage1{}, kt + 1);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);     // the empty loads past the last tile write LDS: none may outlive the workgroup

  // where a pair's results go: the wave's block of the partials, or its row of the output
  const int64_t block = part_block(a, a.part.n_seg, l, slot, g, kWaves, wave, seg);
  auto row_of = [&](int p) -> int64_t {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (p >> lg);
    return tok * a.Hq + g * a.group + (p & (a.group - 1));
  };
  if constexpr (kSplitKeys) {
    if (!idle) {
      float* op = a.part.acc + block * (32 * D) + lane * 4;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<float4*>(op + (d * 4 + r4) * 256) =
              make_float4(o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]);
      if (half == 0) *reinterpret_cast<float2*>(a.part.ml + (block * 32 + lrow) * 2) = make_float2(m, lsum);
    }
  } else {
    fold();
    if (row_ok) {
      const float inv = 1.0f / l_run;
      uint16_t* op = static_cast<uint16_t*>(a.out) + row_of(pair0 + lrow) * D;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<uint2*>(op + d * 32 + r4 * 8 + half * 4) =
              make_uint2(pack_bf16_rne(row_result(o_run[d][r4 * 4], inv), row_result(o_run[d][r4 * 4 + 1], inv)),
                         pack_bf16_rne(row_result(o_run[d][r4 * 4 + 2], inv), row_result(o_run[d][r4 * 4 + 3], inv)));
    }
  }
  // ---- the values that are not finite, to the rows that see them
  __syncthreads();
  if (s_bad != 0 && !idle) {
    __builtin_amdgcn_s_waitcnt(0x0F70);
    const int pairs = min(32, (len << lg) - pair0);
    for (int kt = kt_begin; kt < n_tiles; ++kt) {
      const int key0 = kt * kTileKeys;
      if (!(min(key0 + kTileKeys, n_hi) - 1 > tile_first || key0 < tile_mask_lo)) continue;
      put_bad_values(a, vpool, bt, g, max(key0, wave_lo), min(key0 + kTileKeys, wave_last + 1), W, ctx, lg, pair0, pairs,
                     [&](int p, int x, float v) {
                       if constexpr (kSplitKeys) {
                         float* to = a.part.acc + block * (32 * D) + part_at(p, x);
                         *to = take_in(*to, v);
                       } else {
                         uint16_t* to = static_cast<uint16_t*>(a.out) + row_of(pair0 + p) * D + x;
                         *to = (uint16_t)(__float_as_uint(take_in(bf16_bits_to_f32(*to), v)) >> 16);
                       }
                     });
    }
  }
}

template <typename T, int D>
hipError_t launch_d(const PackedAttnArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)packed_tile_workgroups(a));
  if (a.part.n_seg > 1)
    packed_tiles_kernel<T, D, true><<<grid, 64 * kWaves, 0, stream>>>(a);
  else
    packed_tiles_kernel<T, D, false><<<grid, 64 * kWaves, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const PackedAttnArgs& a, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_d<T, 64>(a, stream);
    case 128: return launch_d<T, 128>(a, stream);
    case 256: return launch_d<T, 256>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_packed_tiles(const PackedAttnArgs& a, int dtype, hipStream_t stream) {
  if (dtype == kDtypeBf16) return launch_t<uint16_t>(a, stream);
  if (dtype == kDtypeFp8) return launch_t<uint8_t>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace kvg
