// Causal attention of packed sequences over int8 caches, on the int8 and fp16 matrix cores.
//
// Workgroup = (layer, KV head g, tile of a sequence): kTilePairs (row, query head) pairs of the sequence, heads fastest, 32 per
// wave.  Keys come in tiles of 64 (absolute multiples of 64 of the logical index) in two LDS stages.
//
// A row's sums have one order, whatever the launch: keys in blocks of 32 (two pages), an online softmax over the blocks of a segment
// of kPackedSeg keys, and the segments' states folded in ascending order (packed_fold_kernel does the same operations).
// References are the row's own (Int8State), so pages that it does not see change nothing.
//
//   S^T = K Q^T     A = K rows from LDS as they are cached (buffer_load ... lds a tile ahead), B = the pairs' queries, two bytes a
//                   value (kvg_int8_mfma.h)
//   O^T += V^T P^T  A = V^T fragments (ds_read_b64_tr_b16), B = P straight from the S^T registers.  V is widened to fp16 on its way:
//                   each wave takes one page of the next tile through registers into LDS, once for the four waves that read it
//                   (widened beside the reads, every wave spent 160 vector instructions a tile of head_dim 128 on it instead of 40)
//
// Bound: vector instructions beside the matrix ones (head_dim 128 has the vector unit busy 66% of the time, the matrix cores 32%; how far the
// two overlap these counters do not say), so the loop is counted in them: ids and scales once a segment, references seldom raised.  Eight prompts of up to 4,096
// tokens, 32 heads on 16, head_dim 128: 540 us (714 TFLOP/s; ids and scales loaded a page at a time 616).  head_dim 256 has one wave a
// SIMD and copies accumulators between the two register files: one prompt of 12,288 tokens, 16 heads on 8, 2.39 ms (518 TFLOP/s).
#include "kvg_int8_mfma.h"
#include "kvg_launch.h"

namespace kvg {

namespace {

constexpr int kTileKeys = 64;
constexpr int kSegTiles = kPackedSeg / kTileKeys, kSegPages = kPackedSeg / kPage;
constexpr int kWaves = 4;
// kSplitKeys: a workgroup takes one segment and leaves its partial.  DV: dimensions of the values that a workgroup sums, all of them or
// half (the scores are then computed twice).  Waves a SIMD are what the registers give; head_dim 64 is held to three, without which the
// compiler takes one register more than they have: 16 prompts of up to 4,096 tokens, 4 heads on 2, 116 us, with two waves 129.
template <int D, int DV, bool kSplitKeys>
__global__ __launch_bounds__(64 * kWaves, DV == 256 ? 1 : D == 64 ? (kSplitKeys ? 4 : 3) : 2) void int8_tiles_kernel(const PackedAttnArgs a, const Int8Scales scales) {
  constexpr int NS = D / 32;               // score steps over head_dim
  constexpr int ND = DV / 32;              // 32-wide blocks of the values' dimensions
  constexpr int kParts = D / DV;
  constexpr int BM = kTilePairs;
  static_assert(BM == 32 * kWaves, "a block of 32 pairs per wave");
  using KR = KRows<D>;
  using VR = VRows<2 * DV>;
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
  const int part = kParts == 1 ? 0 : (int)(id % kParts);
  id /= kParts;
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

  // ---- loads: wave w brings page w of tile kt; rows past the last one the workgroup needs read as zeros.  Lane i has the id and the
  // scales of page i of a segment (its 32 pages), a segment ahead.
  const int source = KR::source(lane);
  int seg_now = kt_begin / kSegTiles;                  // the segment that `pages` is of
  auto pages_of_segment = [&](int sg) -> int32_t {
    const int32_t page = bt[min(sg * kSegPages + (lane & (kSegPages - 1)), last_page)];
    return page >= 0 && page < a.n_pages ? page : 0;
  };
  int32_t pages = pages_of_segment(kt_begin / kSegTiles), pages_next = pages_of_segment(kt_begin / kSegTiles + 1);
  auto slab_of = [&](int kt) -> int64_t {              // of this wave's page of tile kt, which is in this segment or the next
    const int i = kt % kSegTiles * (kTileKeys / kPage) + wave;
    const int32_t here = __builtin_amdgcn_readlane(pages, i), there = __builtin_amdgcn_readlane(pages_next, i);
    return ((int64_t)(kt / kSegTiles == seg_now ? here : there) * a.Hkv + g) * kPage * D;
  };
  auto rows_of = [&](int kt) -> int {
    return __builtin_amdgcn_readfirstlane(min(max(n_hi - (kt * (kTileKeys / kPage) + wave) * kPage, 0), kPage));
  };
  auto issue_k = [&](int kt, auto stage) {
    lds_char* dk = (lds_char*)(lds_void*)((decltype(stage)::value ? sB_K1 : sB_K0) + wave * KR::kPageBytes);
    load_page<KR, 0>(kpool + slab_of(kt), rows_of(kt), dk, source);
  };
  // V: 16 bytes of a row are a lane's.  Its row and place of load j are such that the lanes' stores of widened values lie side by side.
  constexpr int kVLoads = DV / 64;
  constexpr int kLines = VR::kRows;                      // rows whose 16-byte chunks lie side by side
  const int v_row = lane % kLines + lane / 32 * (32 / (DV / 16)), v_col = lane % 32 / kLines;
  const int v_source = v_row * D + part * DV + v_col * 16;
  static_assert(32 / (DV / 16) == kLines, "half a wave takes kLines rows");
  const int v_store = wave * VR::kPageBytes + VR::at(v_row, 2 * v_col);
  constexpr int kNextChunk = VR::at(0, 1), kNextLoad = 2 * VR::kLoad;
  static_assert(1024 / DV == 2 * kLines, "a load takes 2 kLines rows");
  uint4 v_raw[kVLoads];
  auto issue_v = [&](int kt) {
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vpool + slab_of(kt)), 0, rows_of(kt) * D, kBufferWord3);
#pragma unroll
    for (int j = 0; j < kVLoads; ++j) v_raw[j] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, v_source, 2 * kLines * D * j, 0));
  };
  auto widen_v = [&](auto stage, int j) {
    char* to = (decltype(stage)::value ? sA_V1 : sA_V0) + v_store + j * kNextLoad;
    *reinterpret_cast<uint4*>(to) = widen_int8(make_uint2(v_raw[j].x, v_raw[j].y));
    *reinterpret_cast<uint4*>(to + kNextChunk) = widen_int8(make_uint2(v_raw[j].z, v_raw[j].w));
  };

  // ---- queries (B operand of S^T); lanes past the rows take the first row's, and store nothing
  Int8Query<D> q;
  {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (row_ok ? row : 0);
    uint4 raw[NS][2];
    load_query<D>(raw, static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)(g * a.group + ((pair0 + lrow) & (a.group - 1))) * D,
                  half);
    split_query<D>(q, raw);
  }
  const float q_scale = q.step * a.scale_log2;

  const float l0 = q.finite ? 0.0f : kNaN;
  f32x16 o[ND], o_run[kSplitKeys ? 1 : ND];
  Int8State st = empty_state(l0);
  float m_run = -INFINITY, l_run = 0.0f;
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    o[d] = splat(0.0f);
    if constexpr (!kSplitKeys) o_run[d] = splat(0.0f);
  }

  const int k_lane = k_lane_base<D, false>(lane), v_lane = v_lane_base<2 * DV, false>(lane);

  using Stage0 = std::integral_constant<int, 0>;
  using Stage1 = std::integral_constant<int, 1>;
  float ks_next, vs_next;
  auto load_scales = [&](int32_t page) {
    const int64_t at = sbase + (int64_t)page * a.Hkv;
    ks_next = scales.k[at];
    vs_next = scales.v[at];
  };
  issue_v(kt_begin);
  issue_k(kt_begin, Stage0{});
  load_scales(pages);
  PageScales sc = page_scales(ks_next, vs_next);
  uint32_t bad = (uint32_t)__builtin_amdgcn_ballot_w64(sc.bad);
  load_scales(pages_next);
#pragma unroll
  for (int j = 0; j < kVLoads; ++j) widen_v(Stage0{}, j);
  issue_v(kt_begin + 1);

  bool fresh = true;                      // no block of the segment yet
  bool any_far = false;                   // a row of the wave is_far
  auto tile = [&](auto stage, int kt) __attribute__((always_inline)) {
    constexpr int ST = decltype(stage)::value;
    using Next = std::integral_constant<int, 1 - ST>;
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's K of tile kt and V of the next one are here, and what a segment ahead needs
    __syncthreads();                      // all of tile kt is in LDS; the other stage is no longer read
    const int key0 = kt * kTileKeys, page0 = kt % kSegTiles * (kTileKeys / kPage);
    if (kt / kSegTiles != seg_now) {
      ++seg_now;
      pages = pages_next;
      sc = page_scales(ks_next, vs_next);
      bad = (uint32_t)__builtin_amdgcn_ballot_w64(sc.bad);
      pages_next = pages_of_segment(seg_now + 1);
    } else if (kt % kSegTiles == 1) {
      load_scales(pages_next);
    }
    issue_k(kt + 1, Next{});
#pragma unroll
    for (int j = 0; j < kVLoads; ++j) widen_v(Next{}, j);
    issue_v(kt + 2);
    if (key0 > wave_last || key0 + kTileKeys <= wave_lo) return;       // unseen by this wave's rows
    if ((bad >> page0 & 15u) != 0) {
      for (int p = 0; p < kTileKeys / kPage; ++p)
        if ((bad >> (page0 + p) & 1u) != 0 && key0 + p * kPage <= row_n && key0 + (p + 1) * kPage > row_lo) st.l = kNaN;
    }
    const lds_char* kbase = (const lds_char*)(lds_void*)(ST ? sB_K1 : sB_K0) + k_lane;
    const lds_char* vbase = (const lds_char*)(lds_void*)(ST ? sA_V1 : sA_V0) + v_lane;
    const bool need_mask = key0 + kTileKeys - 1 > wave_first || key0 < mask_lo;
    auto kread = [&](int f) { return int8_k_fragment<D>(kbase + KR::at(32 * (f / NS), 0), f % NS); };          // f = block * NS + step
    auto vread = [&](int t) { return v_fragment<2 * DV, false>(vbase + VR::at(16 * (t / ND), 0), t % ND); };    // t = 16-key step * ND + d
    // -Inf where the row does not see the key
    auto mask = [&](f32x16& s, int kb) __attribute__((always_inline)) {
      if (need_mask) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          // key - row_lo as unsigned: keys below the window wrap round
          const uint32_t key = key0 + kb * 32 + half * 4 - row_lo + (r >> 2) * 8 + (r & 3);
          s[r] = key <= (uint32_t)(row_n - row_lo) ? s[r] : -INFINITY;
        }
      }
    };
    // the references of block kb from a lane's largest scores of its pages, O and the sum of p with them (O of a segment's first block
    // is still 0)
    auto references = [&](float mx0, float mx1, float kq0, float kq1, float lv0, float lv1) __attribute__((always_inline)) {
      const float2 mx = max_halves(mx0, mx1);
      const float t0 = largest_score(mx.x, kq0), t1 = largest_score(mx.y, kq1);
      const bool raised = is_raised(st, t0, t1, lv0, lv1);
      if (__builtin_amdgcn_ballot_w64(raised) != 0) {                                // seldom: the references are coarse
        const Int8Raise up = raise_block(st, raised, t0, t1, lv0, lv1);
        any_far = __builtin_amdgcn_ballot_w64(is_far(st)) != 0;
        st.l *= up.alpha_l;
        if (!fresh) {
#pragma unroll
          for (int d = 0; d < ND; ++d) o[d] *= up.alpha_o;
        }
      }
      fresh = false;
    };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float kq0 = key_factor(q_scale, lane_value(sc.k, page0 + 2 * kb)), kq1 = key_factor(q_scale, lane_value(sc.k, page0 + 2 * kb + 1));
      const float lv0 = lane_value(sc.lv, page0 + 2 * kb), lv1 = lane_value(sc.lv, page0 + 2 * kb + 1);
      uint4 kf[NS];
#pragma unroll
      for (int ss = 0; ss < NS; ++ss) kf[ss] = kread(kb * NS + ss);
      // the queries' upper bytes, then the lower ones on top of 256 times their sums
      i32x16 acc = (i32x16)(0);
#pragma unroll
      for (int ss = 0; ss < NS; ++ss) acc = mfma_i8(kf[ss], q.hi[ss], acc);
      acc <<= 8;
#pragma unroll
      for (int ss = 0; ss < NS; ++ss) acc = mfma_i8(kf[ss], q.lo[ss], acc);
      f32x16 s = __builtin_convertvector(acc, f32x16);
      mask(s, kb);
      float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        mx0 = fmaxf(mx0, s[r]);
        mx1 = fmaxf(mx1, s[8 + r]);
      }
      references(mx0, mx1, kq0, kq1, lv0, lv1);
      Int8Page p0 = page_weights(st, lv0), p1 = page_weights(st, lv1);
      if (any_far) {
        far_page(s, 0, kq0, p0, st, lv0);
        far_page(s, 8, kq1, p1, st, lv1);
      }
      float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        s[r] = weight_of(s[r], kq0, p0.c);
        sum0 += s[r];
      }
#pragma unroll
      for (int r = 8; r < 16; ++r) {
        s[r] = weight_of(s[r], kq1, p1.c);
        sum1 += s[r];
      }
      const uint4 w0 = round_weights8(s, 0), w1 = round_weights8(s, 1);
      st.l += block_sum(sum0, sum1, p0.back, p1.back);
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = mfma_f16(vread(kb * 2 * ND + d), w0, o[d]);
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = mfma_f16(vread(kb * 2 * ND + ND + d), w1, o[d]);
    }
  };
  // end of a segment: its sums taken to the reference of p, its state folded into the running one, which packed_fold_kernel does with
  // the same operations (the power of two in the factor would round sums below fp32's range otherwise)
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
      st = empty_state(l0);
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = splat(0.0f);
      fresh = true;
      any_far = false;
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
    float* op = a.part.acc + block * (32 * D) + part * (32 * DV) + lane * 4;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<float4*>(op + (d * 4 + r4) * 256) =
            make_float4(o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]);
    if (half == 0 && part == 0) *reinterpret_cast<float2*>(a.part.ml + (block * 32 + lrow) * 2) = make_float2(st.m, st.l);
  } else {
    fold();
    if (!row_ok) return;
    const float inv = 1.0f / l_run;
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + row;
    uint16_t* op = static_cast<uint16_t*>(a.out) + (tok * a.Hq + g * a.group + ((pair0 + lrow) & (a.group - 1))) * D + part * DV;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<uint2*>(op + d * 32 + r4 * 8 + half * 4) =
            make_uint2(pack_bf16_rne(row_result(o_run[d][r4 * 4], inv), row_result(o_run[d][r4 * 4 + 1], inv)),
                       pack_bf16_rne(row_result(o_run[d][r4 * 4 + 2], inv), row_result(o_run[d][r4 * 4 + 3], inv)));
  }
}

template <int D>
hipError_t launch_d(const PackedAttnArgs& a, const Int8Scales& s, hipStream_t stream) {
  const int64_t grid = packed_tile_workgroups(a);
  // Where the running sums of the segments are not held, half of 256 dimensions lets two workgroups share a compute unit: 512 tokens over
  // 4,096 99 us (with all of them 112), 4 x 35 over 32,768 164 (169).
  if (a.part.n_seg > 1) {
    constexpr int DV = int8_split_values(D);
    int8_tiles_kernel<D, DV, true><<<(unsigned)(grid * (D / DV)), 64 * kWaves, 0, stream>>>(a, s);
  } else {
    int8_tiles_kernel<D, D, false><<<(unsigned)grid, 64 * kWaves, 0, stream>>>(a, s);
  }
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
