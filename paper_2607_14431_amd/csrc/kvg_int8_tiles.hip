// Causal attention of packed sequences over int8 caches, on the int8 and fp16 matrix cores.
//
// Workgroup = (layer, KV head g, tile of a sequence): kTilePairs (row, query head) pairs of the sequence, heads fastest, 32 per
// wave.  Keys come in tiles of 64 (absolute multiples of 64 of the logical index) in two LDS stages, loaded with
// buffer_load ... lds while the tile before is computed.
//
// A row's sums have one order, whatever the launch: keys in blocks of 32 (two pages), an online softmax over the blocks of a segment
// of kPackedSeg keys, and the segments' states folded in ascending order (packed_fold_kernel does the same operations).
// References are the row's own (Int8State), so pages that it does not see change nothing.
//
//   S^T = K Q^T     A = K rows from LDS as they are cached, B = the pairs' queries, two bytes a value (kvg_int8_mfma.h)
//   O^T += V^T P^T  A = V^T fragments (ds_read_b64_tr_b8) widened to fp16, B = P straight from the S^T registers
#include "kvg_int8_mfma.h"
#include "kvg_launch.h"

#include <type_traits>

namespace kvg {

namespace {

constexpr int kTileKeys = 64;
constexpr int kSegTiles = kPackedSeg / kTileKeys;
constexpr int kWaves = 4;
// kSplitKeys: a workgroup takes one segment and leaves its partial.
template <int D, bool kSplitKeys>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void int8_tiles_kernel(const PackedAttnArgs a, const Int8Scales scales) {
  constexpr int NS = D / 32;               // score steps over head_dim
  constexpr int ND = D / 32;               // 32-wide blocks of head_dim
  constexpr int BM = kTilePairs;
  static_assert(BM == 32 * kWaves, "a block of 32 pairs per wave");
  using KR = KRows<D>;
  using VR = VRows<D>;
  // a wave brings one page of a tile; the V stages first, where an LDS instruction's immediate offset reaches
  __shared__ __attribute__((aligned(1024))) char sA_V0[kWaves * VR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char sA_V1[kWaves * VR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char sB_K0[kWaves * KR::kPageBytes];
  __shared__ __attribute__((aligned(1024))) char sB_K1[kWaves * KR::kPageBytes];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int lrow = lane & 31, half = lane >> 5;
  const int lg = 31 - __builtin_clz(a.group);            // 1, 2, 4 or 8 query heads per KV head

  // ---- (tile, layer, segment, KV head), the KV head fastest; late tiles, which have the most keys, first (as packed_tiles_kernel)
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
  if constexpr (kSplitKeys) seg = (int)((uint32_t)(seg + slot) % (uint32_t)a.part.n_seg);
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
  const char* kpool = static_cast<const char*>(a.k_pool) + lbase;
  const char* vpool = static_cast<const char*>(a.v_pool) + lbase;
  const int64_t sbase = (int64_t)(a.layer0 + l) * a.n_pages * a.Hkv + g;

  // ---- loads: wave w brings page w of tile kt; rows past the last one the workgroup needs read as zeros.  Lane i has the id of page
  // i % 4 of a tile and, a tile later, its scales.
  const int source = KR::source(lane);     // the same for V
  auto pages_of_tile = [&](int kt) -> int32_t {
    const int32_t page = bt[min(kt * (kTileKeys / kPage) + (lane & 3), last_page)];
    return page >= 0 && page < a.n_pages ? page : 0;
  };
  constexpr int kTileLoads = 2 * KR::kPageLoads;       // of a wave: K and V alternate
  auto issue = [&](int kt, int32_t pages, auto dst_stage, int j0, int j1) {
    constexpr int DS = decltype(dst_stage)::value;
    const int64_t off = ((int64_t)__builtin_amdgcn_readlane(pages, wave) * a.Hkv + g) * kPage * D;
    const int rows = __builtin_amdgcn_readfirstlane(min(max(n_hi - (kt * (kTileKeys / kPage) + wave) * kPage, 0), kPage));
    lds_char* dk = (lds_char*)(lds_void*)((DS ? sB_K1 : sB_K0) + wave * KR::kPageBytes);
    lds_char* dv = (lds_char*)(lds_void*)((DS ? sA_V1 : sA_V0) + wave * VR::kPageBytes);
    load_page<KR, 0>(kpool + off, rows, dk, source, (j0 + 1) / 2, (j1 + 1) / 2);
    load_page<VR, 0>(vpool + off, rows, dv, source, j0 / 2, j1 / 2);
  };

  // ---- queries (B operand of S^T), zeros past the rows
  Int8Query<D> q;
  {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (row_ok ? row : 0);
    load_query<D>(q, static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)(g * a.group + ((pair0 + lrow) & (a.group - 1))) * D,
                  row_ok, half);
  }
  const float q_scale = q.step * a.scale_log2;

  f32x16 o[ND], o_run[kSplitKeys ? 1 : ND];
  Int8State st = {-INFINITY, -INFINITY, 0.0f};
  float m_run = -INFINITY, l_run = 0.0f;
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    o[d] = splat(0.0f);
    if constexpr (!kSplitKeys) o_run[d] = splat(0.0f);
  }

  const int k_lane = k_lane_base<D, false>(lane), v_lane = v_lane_base<D, true>(lane);

  using Stage0 = std::integral_constant<int, 0>;
  using Stage1 = std::integral_constant<int, 1>;
  int32_t pages_next = pages_of_tile(kt_begin);
  float ks_next = scales.k[sbase + (int64_t)pages_next * a.Hkv], vs_next = scales.v[sbase + (int64_t)pages_next * a.Hkv];
  issue(kt_begin, pages_next, Stage0{}, 0, kTileLoads);
  pages_next = pages_of_tile(kt_begin + 1);

  bool fresh = true;                      // no block of the segment yet
  auto tile = [&](auto stage, int kt) __attribute__((always_inline)) {
    constexpr int ST = decltype(stage)::value;
    using Next = std::integral_constant<int, 1 - ST>;
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's share of tile kt, its scales and the next page ids are here
    __syncthreads();                      // all of tile kt is in LDS; the other stage is no longer read
    const int key0 = kt * kTileKeys;
    const float ks = ks_next, vs = vs_next;
    const int32_t pages = pages_next;
    ks_next = scales.k[sbase + (int64_t)pages * a.Hkv];
    vs_next = scales.v[sbase + (int64_t)pages * a.Hkv];
    pages_next = pages_of_tile(kt + 2);
    issue(kt + 1, pages, Next{}, 0, kTileLoads);
    if (key0 > wave_last || key0 + kTileKeys <= wave_lo) return;       // unseen by this wave's rows
    const lds_char* kbase = (const lds_char*)(lds_void*)(ST ? sB_K1 : sB_K0) + k_lane;
    const lds_char* vbase = (const lds_char*)(lds_void*)(ST ? sA_V1 : sA_V0) + v_lane;
    const bool need_mask = key0 + kTileKeys - 1 > wave_first || key0 < mask_lo;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      i32x16 hi = (i32x16)(0), lo = (i32x16)(0);
#pragma unroll
      for (int ss = 0; ss < NS; ++ss) {
        const uint4 k = int8_k_fragment<D>(kbase + KR::at(32 * kb, 0), ss);
        hi = mfma_i8(k, q.hi[ss], hi);
        lo = mfma_i8(k, q.lo[ss], lo);
      }
      auto scales_of = [&](int p) -> PageScales {
        return page_scales(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), p)),
                           __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), p)));
      };
      const PageScales p0 = scales_of(2 * kb), p1 = scales_of(2 * kb + 1);
      f32x16 s = int8_scores(hi, lo, q_scale * p0.k, q_scale * p1.k);
      if (need_mask) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // key - row_lo as unsigned: keys below the window wrap round
          const uint32_t key = key0 + kb * 32 + half * 4 - row_lo + (r >> 2) * 8 + (r & 3);
          s[r] = key <= (uint32_t)(row_n - row_lo) ? s[r] : -INFINITY;
        }
      }
      const float2 mx = page_maxima(s);
      const Int8Block blk = raise_block(st, mx.x, mx.y, p0, p1);
      uint4 p[2];
      st.l = fmaf(st.l, blk.alpha_l, block_weights(s, blk, p));
      if (!fresh && __builtin_amdgcn_ballot_w64(blk.raised) != 0) {    // O of a segment's first block is still 0
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= blk.alpha_o;
      }
      fresh = false;
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i)
        o[i % ND] = mfma_f16(widen_int8(v_fragment<D, true>(vbase + VR::at(32 * kb + 16 * (i / ND), 0), i % ND)), p[i / ND], o[i % ND]);
    }
  };
  // end of a segment: its sums at the reference of the exponentials; its state folded into the running one, which
  // packed_fold_kernel does with the same operations
  auto end_segment = [&]() {
    const int e = end_exponent(st);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = __builtin_ldexpf(o[d][r], e);
  };
  auto fold = [&]() {
    if constexpr (!kSplitKeys) {
      end_segment();
      const FoldFactors f = fold_factors(m_run, l_run, st.m, st.l);
#pragma unroll
      for (int d = 0; d < ND; ++d) o_run[d] = __builtin_elementwise_fma(o[d], splat(f.part), o_run[d] * f.run);
      st = {-INFINITY, -INFINITY, 0.0f};
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

  if constexpr (kSplitKeys) {
    if (idle) return;
    end_segment();
    const int64_t block = part_block(a, a.part.n_seg, l, slot, g, kWaves, wave, seg);
    float* op = a.part.acc + block * (32 * D) + lane * 4;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<float4*>(op + (d * 4 + r4) * 256) =
            make_float4(o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]);
    if (half == 0) *reinterpret_cast<float2*>(a.part.ml + (block * 32 + lrow) * 2) = make_float2(st.m, st.l);
  } else {
    fold();
    if (!row_ok) return;
    const float inv = 1.0f / l_run;
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + row;
    uint16_t* op = static_cast<uint16_t*>(a.out) + (tok * a.Hq + g * a.group + ((pair0 + lrow) & (a.group - 1))) * D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<uint2*>(op + d * 32 + r4 * 8 + half * 4) =
            make_uint2(pack_bf16_rne(o_run[d][r4 * 4] * inv, o_run[d][r4 * 4 + 1] * inv),
                       pack_bf16_rne(o_run[d][r4 * 4 + 2] * inv, o_run[d][r4 * 4 + 3] * inv));
  }
}

template <int D>
hipError_t launch_d(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream) {
  const dim3 grid((unsigned)packed_tile_workgroups(a));
  if (a.part.n_seg > 1)
    int8_tiles_kernel<D, true><<<grid, 64 * kWaves, 0, stream>>>(a, s);
  else
    int8_tiles_kernel<D, false><<<grid, 64 * kWaves, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_int8_tiles(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_d<64>(a, s, stream);
    case 128: return launch_d<128>(a, s, stream);
    case 256: return launch_d<256>(a, s, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvg
