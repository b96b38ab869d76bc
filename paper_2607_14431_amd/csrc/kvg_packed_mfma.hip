// Causal attention of packed sequences over a paged bf16 or fp8 cache, on bf16 MFMA (v_mfma_f32_32x32x16_bf16).
//
// Workgroup = (layer, KV head g, tile of a sequence): BM (row, query head) pairs of the sequence, heads
// fastest, kBlocks blocks of 32 pairs per wave.  Keys come in tiles of 64 (absolute multiples of 64 of the
// logical index) in two LDS stages, loaded with buffer_load ... lds while the tile before is computed.
//
// A row's sums have one order, whatever the launch: keys in blocks of 32, an online softmax over the blocks of a
// segment of kSeg keys (absolute multiples), and the segments' states folded in ascending order.  A
// workgroup that walks all keys folds in registers; split launches leave one partial per segment for
// packed_fold_kernel, which folds them with the same operations.
//
//   S^T = K Q^T    A = K rows from LDS, B = the pairs' queries in registers; a lane owns one pair (lane % 32) and 16
//                  of a block's 32 keys, the other 16 are in lane ^ 32
//   softmax        fp32; the reference is the largest score rounded up to a multiple of kStep in log2 units and moves
//                  only when a block exceeds it, so states of different segments mostly share it and
//                  fold by one addition; weights are rounded to bf16 and summed as rounded, so a row of one key
//                  gives its value exactly and rounding errors of the heavy weights cancel
//   O^T += V^T P^T A = V^T fragments (ds_read_b64_tr), B = P straight from the S^T registers
#include "kvg_launch.h"
#include "kvg_mfma.h"
#include "kvg_packed.h"
#include "kvg_rows.h"

#include <math.h>

#include <type_traits>

namespace kvg {

namespace {

constexpr int kTileKeys = 64;
constexpr int kSegTiles = kPackedSeg / kTileKeys;
constexpr int kWaves = 4;
constexpr float kStep = 8.0f;          // grid of the references, log2 units

// The reference that a largest score (log2 units) asks for.
__device__ __forceinline__ float reference_of(float mx) { return ceilf(mx * (1.0f / kStep)) * kStep; }

// LDS rows hold their 16-byte chunks at position chunk ^ swizzle(row), XOR-linear in the row bits.  K is read as one chunk
// of 32 consecutive rows per lane half, V transposed (bf16: four rows x two or four chunks, fp8: rows
// {0..3, 8..11} (+ 4) of a 16-row step).
template <int RB, bool kFp8>
struct SwzTile {
  __device__ static __forceinline__ int k(int r) {
    if constexpr (kFp8) return RB == 256 ? (r & 15) : RB == 128 ? ((r >> 1) & 7) : ((r >> 2) & 3);
    return RB >= 256 ? (r & 15) : (r & 7);
  }
  __device__ static __forceinline__ int v(int r) {
    if constexpr (kFp8)
      return RB == 256 ? (r & 15) : RB == 128 ? (((r >> 1) & 1) | (((r >> 3) & 1) << 1)) : ((r >> 3) & 1);
    return RB >= 256 ? ((0xCA60 >> (4 * (r & 3))) & 15) : 2 * (r & 3);
  }
};

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
template <typename T, int NCH>
__device__ __forceinline__ bool finite_rows(uint4* p, int lane) {
  bool any = false;
#pragma unroll 2
  for (int i = lane; i < kPage * NCH; i += 64) {
    uint4 x = p[i];
    if (!bad_values(x, T{})) continue;
    any = true;
    T* v = reinterpret_cast<T*>(p + i);
    for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
      if (!(fabsf(load_value(v + e)) < INFINITY)) v[e] = 0;
  }
  return __builtin_amdgcn_ballot_w64(any) != 0;
}

__device__ __forceinline__ f32x16 splat(float x) { return (f32x16)(x); }

// T: cache storage (uint16_t bf16, uint8_t fp8 E4M3).  kBlocks: blocks of 32 pairs per wave.
// kSplit: a workgroup takes one segment and leaves its partial.
template <typename T, int D, int kBlocks, bool kSplitKeys>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void packed_mfma_kernel(const PackedAttnArgs a) {
  constexpr bool kFp8 = sizeof(T) == 1;
  constexpr int RB = D * (int)sizeof(T);   // bytes per cache row
  constexpr int NCH = RB / 16;             // 16-byte chunks per row
  constexpr int NS = D / 16;               // MFMA steps over head_dim
  constexpr int ND = D / 32;               // 32-wide blocks of head_dim
  constexpr int kTileChunks = kTileKeys * NCH;
  constexpr int kLoads = NCH / kWaves;     // direct loads per lane and operand: a wave brings one page of the tile
  constexpr int BM = 32 * kBlocks * kWaves;
  using SW = SwzTile<RB, kFp8>;
  __shared__ __attribute__((aligned(1024))) uint4 sA_V0[kTileChunks];
  __shared__ __attribute__((aligned(1024))) uint4 sA_V1[kTileChunks];
  __shared__ __attribute__((aligned(1024))) uint4 sB_K0[kTileChunks];
  __shared__ __attribute__((aligned(1024))) uint4 sB_K1[kTileChunks];
  __shared__ int s_bad;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int lrow = lane & 31, half = lane >> 5;
  const int lg = 31 - __builtin_clz(a.group);            // 1, 2, 4 or 8 query heads per KV head

  // ---- (layer, segment, tile, KV head), the KV head fastest; late tiles, which have the most keys, first
  uint32_t id = blockIdx.x;
  const int g = (int)(id % (uint32_t)a.Hkv);
  id /= (uint32_t)a.Hkv;
  const int slot = (int)(id % (uint32_t)a.n_tiles);
  id /= (uint32_t)a.n_tiles;
  int seg = 0;
  if constexpr (kSplitKeys) {
    seg = (int)(id % (uint32_t)a.n_seg);
    id /= (uint32_t)a.n_seg;
  }
  const int l = (int)id;
  const SeqUnit u = find_unit(a.seqs, slot, [&](const SeqRange& s) { return (int)((((int64_t)s.len << lg) + BM - 1) / BM); });
  if (u.b < 0) return;
  const SeqRange sq = u.range;
  const int tile_id = u.count - 1 - u.at;
  const int ctx = sq.ctx, len = sq.len;

  const int pair0 = tile_id * BM + wave * (32 * kBlocks);   // this wave's first pair
  int row_n[kBlocks], row_lo[kBlocks];                      // this lane's rows' visible keys [row_lo, row_n]
  bool row_ok[kBlocks];
  const int W = layer_window(a, l);
#pragma unroll
  for (int rb = 0; rb < kBlocks; ++rb) {
    const int row = (pair0 + 32 * rb + lrow) >> lg;
    row_ok[rb] = row < len;
    row_n[rb] = ctx + row;
    row_lo[rb] = window_start(W, ctx + row + 1);
  }
  const int first_row = pair0 >> lg;
  const int last_row = min((pair0 + 32 * kBlocks - 1) >> lg, len - 1);
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

  // ---- loads: wave w brings page w of tile kt (rows 16 w ..).  Instruction i covers slots [64 i, 64 i + 64) of the page's
  // rows: row (64 i + lane) / NCH, position (64 i + lane) % NCH.  The resource over a (page, head) slab ends
  // at the last row the workgroup needs: rows past it read as zeros.
  constexpr int kRowsPerLoad = 64 / NCH;
  const int lrow0 = lane / NCH;
  const uint32_t k_off0 = lrow0 * RB + 16 * ((lane % NCH) ^ SW::k(lrow0));
  const uint32_t v_off0 = lrow0 * RB + 16 * ((lane % NCH) ^ SW::v(lrow0));
  auto page_slot = [&](int kt) { return kt * (kTileKeys / kPage) + wave; };
  auto page_of_tile = [&](int kt) -> int32_t { return bt[min(page_slot(kt), last_page)]; };
  auto tile_rsrc = [&](const T* pool, int kt, int32_t page) {
    page = __builtin_amdgcn_readfirstlane(page);
    page = (page >= 0 && page < a.n_pages) ? page : 0;
    const int64_t poff = ((int64_t)page * a.Hkv + g) * kPage * D;
    const int rows = __builtin_amdgcn_readfirstlane(min(max(n_hi - page_slot(kt) * kPage, 0), kPage));
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(pool + poff), 0, rows * RB, kBufferWord3);
  };
  constexpr int kTileLoads = 2 * kLoads;
  auto issue = [&](__amdgpu_buffer_rsrc_t rk, __amdgpu_buffer_rsrc_t rv, auto dst_stage, int j0, int j1) {
    constexpr int DS = decltype(dst_stage)::value;
    lds_char* dk = (lds_char*)(lds_void*)&(DS ? sB_K1 : sB_K0)[wave * kPage * NCH];
    lds_char* dv = (lds_char*)(lds_void*)&(DS ? sA_V1 : sA_V0)[wave * kPage * NCH];
#pragma unroll
    for (int j = j0; j < j1; ++j) {
      const int i = j >> 1;
      if (j & 1) {
        const uint32_t ov = 1024 * i + (v_off0 ^ (16 * SW::v(i * kRowsPerLoad)));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void*)(dv + 1024 * i), 16, ov, 0, 0, 0);
      } else {
        const uint32_t ok = 1024 * i + (k_off0 ^ (16 * SW::k(i * kRowsPerLoad)));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void*)(dk + 1024 * i), 16, ok, 0, 0, 0);
      }
    }
  };

  // ---- queries (B operand of S^T), zeros past the rows
  uint4 qf[kBlocks][NS];
#pragma unroll
  for (int rb = 0; rb < kBlocks; ++rb) {
    const int p = pair0 + 32 * rb + lrow;
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (row_ok[rb] ? p >> lg : 0);
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + tok * a.q_stride + (int64_t)(g * a.group + (p & (a.group - 1))) * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[rb][s] = row_ok[rb] ? ld16(qp + (2 * s + half) * 8) : make_uint4(0, 0, 0, 0);
  }

  f32x16 o[kBlocks][ND], o_run[kSplitKeys ? 1 : kBlocks][ND];
  float m[kBlocks], lsum[kBlocks], m_run[kBlocks], l_run[kBlocks];
#pragma unroll
  for (int rb = 0; rb < kBlocks; ++rb) {
    m[rb] = m_run[rb] = -INFINITY;
    lsum[rb] = l_run[rb] = 0.0f;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      o[rb][d] = splat(0.0f);
      if constexpr (!kSplitKeys) o_run[rb][d] = splat(0.0f);
    }
  }

  // ---- LDS addressing (row base and chunk; a constant XORed into the chunk bits permutes a row's chunks)
  //   K step ss of block kb: row kb * 32 + lrow, chunk 2 ss + half (fp8: 8 bytes at 16 ss + 8 half)
  //   V^T step (ks, d), 16 keys: 16-lane group tr_m = lane / 16, tr_k = lane % 16: bf16 rows 4 (tr_m / 2) + tr_k / 4 (and 8
  //   further), 8 bytes at dim 32 d + 16 (tr_m % 2) + 4 (tr_k % 4); fp8 row 4 (tr_m / 2) + {0..3, 8..11}[tr_k / 2], 8 bytes
  //   at dim 32 d + 16 (tr_m % 2) + 8 (tr_k % 2)
  const int tr_k = lane & 15, tr_m = lane >> 4;
  uint32_t k_lane, v_lane;
  if constexpr (kFp8) {
    const int kk = 4 * (tr_m >> 1) + ((tr_k >> 1) & 3) + 8 * (tr_k >> 3);
    k_lane = lrow * RB + 16 * SW::k(lrow) + 8 * half;
    v_lane = kk * RB + 16 * ((tr_m & 1) ^ SW::v(kk)) + 8 * (tr_k & 1);
  } else {
    const int rr = (tr_m >> 1) * 4 + (tr_k >> 2);
    k_lane = lrow * RB + 16 * (half ^ SW::k(lrow));
    v_lane = rr * RB + 8 * (tr_k & 1) + 16 * ((2 * (tr_m & 1) + ((tr_k & 3) >> 1)) ^ SW::v(rr));
  }

  if (tid == 0) s_bad = 0;              // read and written behind the first tile's barrier
  using Stage0 = std::integral_constant<int, 0>;
  using Stage1 = std::integral_constant<int, 1>;
  int32_t pg_next = page_of_tile(kt_begin);
  issue(tile_rsrc(kpool, kt_begin, pg_next), tile_rsrc(vpool, kt_begin, pg_next), Stage0{}, 0, kTileLoads);
  pg_next = page_of_tile(kt_begin + 1);

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
      if (finite_rows<T, NCH>((ST ? sA_V1 : sA_V0) + wave * kPage * NCH, lane)) s_bad = 1;
      __syncthreads();
    }
    const __amdgpu_buffer_rsrc_t nk = tile_rsrc(kpool, kt + 1, pg_next), nv = tile_rsrc(vpool, kt + 1, pg_next);
    pg_next = page_of_tile(kt + 2);
    if (key0 > wave_last || key0 + kTileKeys <= wave_lo) {       // no row of this wave sees the tile
      issue(nk, nv, Next{}, 0, kTileLoads);
      return;
    }
    // loads of step t (0 <= t < 2 NS over phases A and B)
    auto issue_step = [&](int t) {
      issue(nk, nv, Next{}, t * kTileLoads / (2 * NS), (t + 1) * kTileLoads / (2 * NS));
    };
    const lds_char* kbase = (const lds_char*)(lds_void*)(ST ? sB_K1 : sB_K0);
    const lds_char* vbase = (const lds_char*)(lds_void*)(ST ? sA_V1 : sA_V0);
    auto kread = [&](int f) -> uint4 {    // fragment f = kb * NS + ss
      const int kb = f / NS, ss = f % NS;
      if constexpr (kFp8) {
        const u32x2 w = *reinterpret_cast<const lds_u32x2*>(kbase + (k_lane ^ (uint32_t)(16 * ss)) + kb * 32 * RB);
        return widen_fp8x8(w.x, w.y);
      } else {
        return __builtin_bit_cast(uint4, *reinterpret_cast<const lds_u32x4*>(kbase + (k_lane ^ (uint32_t)(32 * ss)) + kb * 32 * RB));
      }
    };
    auto vread = [&](int t) -> uint4 {    // fragment t = ks * ND + d
      const int ks = t / ND, d = t % ND;
      if constexpr (kFp8) {
        const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vbase + (v_lane ^ (uint32_t)(32 * d)) + ks * 16 * RB));
        return widen_fp8x8((uint32_t)w.x, (uint32_t)w.y);
      } else {
        const uint32_t at = (v_lane ^ (uint32_t)(64 * d)) + ks * 16 * RB;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vbase + at));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vbase + at + 8 * RB));
        const uint2 lo2 = __builtin_bit_cast(uint2, lo), hi2 = __builtin_bit_cast(uint2, hi);
        return make_uint4(lo2.x, lo2.y, hi2.x, hi2.y);
      }
    };

    f32x16 s[2][kBlocks];
    if constexpr (D > 128) {
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb) s[0][rb] = s[1][rb] = splat(0.0f);
    }
    const bool need_mask = key0 + kTileKeys - 1 > wave_first || key0 < mask_lo;
    auto mask_block = [&](int kb) {
      if (need_mask) {
#pragma unroll
        for (int rb = 0; rb < kBlocks; ++rb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = key0 + kb * 32 + half * 4 + (r >> 2) * 8 + (r & 3);
            const int at = D <= 128 ? 0 : kb;
            s[at][rb][r] = (key <= row_n[rb] && key >= row_lo[rb]) ? s[at][rb][r] : -INFINITY;
          }
      }
    };
    // softmax of one block of one row block in 16 pieces, to sit beside the matrix steps of another phase: 0-3 the largest
    // score, 4 the reference, 5-12 two exponentials each, 13-14 rounding of eight weights and their sum, 15 the sum
    uint4 pf[2][kBlocks][2];
    struct SoftState {
      float mx, alpha, m_ref, psum;
      bool raised;
    } st[kBlocks];
    auto soft_piece = [&](int kb, int rb, int j) {
      SoftState& x = st[rb];
      if (j < 4) {
        if (j == 0) x.mx = -INFINITY;
#pragma unroll
        for (int r = 4 * j; r < 4 * j + 4; ++r) x.mx = fmaxf(x.mx, s[kb][rb][r]);
      } else if (j == 4) {
        const float2 mh = halves32(x.mx);
        const float mx = fmaxf(mh.x, mh.y) * a.scale_log2;
        x.raised = mx > m[rb];
        const float up = reference_of(mx);
        x.alpha = x.raised ? __builtin_amdgcn_exp2f(m[rb] - up) : 1.0f;
        m[rb] = x.raised ? up : m[rb];
        x.m_ref = m[rb] == -INFINITY ? 0.0f : m[rb];      // no key seen yet: every weight is 0
        x.psum = 0.0f;
      } else if (j < 13) {
#pragma unroll
        for (int r = 2 * (j - 5); r < 2 * (j - 5) + 2; ++r)
          s[kb][rb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][rb][r], a.scale_log2, -x.m_ref));
      } else if (j < 15) {
        const int hs = j - 13;
        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
        uint4& f = pf[kb][rb][hs];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          (&f.x)[w] = pack_bf16_rne(s[kb][rb][8 * hs + 2 * w], s[kb][rb][8 * hs + 2 * w + 1]);
          x.psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (&f.x)[w]), ones, x.psum, false);
        }
      } else {
        const float2 ph = halves32(x.psum);
        lsum[rb] = lsum[rb] * x.alpha + (ph.x + ph.y);
      }
    };
    auto rescale_o = [&]() {
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb)
        if (__builtin_amdgcn_ballot_w64(st[rb].raised) != 0) {
#pragma unroll
          for (int d = 0; d < ND; ++d) o[rb][d] *= st[rb].alpha;
        }
    };
    auto mfma = [](const uint4& x, const uint4& y, const f32x16& c) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(x), as_bf16x8(y), c, 0, 0, 0);
    };

    // K fragments of both blocks form one stream read LK ahead of their MFMAs, V^T fragments one read LV ahead, whose first
    // LV are issued with block 1's scores
    if constexpr (D <= 128) {
      // two waves a SIMD: one's softmax runs beside the other's matrix steps
      constexpr int LF = 2, RF = LF + 1;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        uint4 kf[RF], vf[RF];
#pragma unroll
        for (int f = 0; f < LF; ++f) kf[f] = kread(kb * NS + f);
#pragma unroll
        for (int ss = 0; ss < NS; ++ss) {
          if (ss + LF < NS) kf[(ss + LF) % RF] = kread(kb * NS + ss + LF);
          issue_step(kb * NS + ss);
#pragma unroll
          for (int rb = 0; rb < kBlocks; ++rb) s[0][rb] = ss ? mfma(kf[ss % RF], qf[rb][ss], s[0][rb]) : mfma(kf[0], qf[rb][0], splat(0.0f));
        }
        mask_block(kb);
        auto vget = [&](int t) { return vread(kb * 2 * ND + t); };
#pragma unroll
        for (int f = 0; f < LF; ++f) vf[f] = vget(f);
#pragma unroll
        for (int rb = 0; rb < kBlocks; ++rb)
#pragma unroll
          for (int j = 0; j < 16; ++j) soft_piece(0, rb, j);
        rescale_o();
#pragma unroll
        for (int t = 0; t < 2 * ND; ++t) {
          if (t + LF < 2 * ND) vf[(t + LF) % RF] = vget(t + LF);
#pragma unroll
          for (int rb = 0; rb < kBlocks; ++rb) o[rb][t % ND] = mfma(vf[t % RF], pf[0][rb][t / ND], o[rb][t % ND]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      return;
    }
    constexpr int LK = 4;
    constexpr int RK = LK + 1;
    constexpr int NT = 4 * ND;
    constexpr int LV = 4;
    constexpr int RV = LV + 1;
    uint4 kf[RK], vf[RV];
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
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb) s[0][rb] = mfma(kf[ss % RK], qf[rb][ss], s[0][rb]);
      __builtin_amdgcn_sched_barrier(0);
    }
    mask_block(0);
    // phase B: scores of block 1 beside the softmax of block 0
    constexpr int kPieces = 16 * kBlocks;
    static_assert(D <= 128 || LV <= NS, "first V^T fragments");
#pragma unroll
    for (int ss = 0; ss < NS; ++ss) {
      const int f = NS + ss;
      kfetch(f + LK);
      issue_step(NS + ss);
      if (ss >= NS - LV) vfetch(ss - (NS - LV));
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb) s[1][rb] = mfma(kf[f % RK], qf[rb][ss], s[1][rb]);
#pragma unroll
      for (int j = ss * kPieces / NS; j < (ss + 1) * kPieces / NS; ++j) soft_piece(0, j % kBlocks, j / kBlocks);
      __builtin_amdgcn_sched_barrier(0);
    }
    rescale_o();
    mask_block(1);
    // phases C and D: O^T += V^T P^T over block 0, beside the softmax of block 1, and over block 1
#pragma unroll
    for (int t = 0; t < 2 * ND; ++t) {
      vfetch(t + LV);
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb) o[rb][t % ND] = mfma(vf[t % RV], pf[0][rb][t / ND], o[rb][t % ND]);
#pragma unroll
      for (int j = t * kPieces / (2 * ND); j < (t + 1) * kPieces / (2 * ND); ++j) soft_piece(1, j % kBlocks, j / kBlocks);
      __builtin_amdgcn_sched_barrier(0);
    }
    rescale_o();
#pragma unroll
    for (int t = 2 * ND; t < NT; ++t) {
      vfetch(t + LV);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb) o[rb][t % ND] = mfma(vf[t % RV], pf[1][rb][t / ND - 2], o[rb][t % ND]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // end of a segment: its state folded into the running one, which packed_fold_kernel does with the same operations
  auto fold = [&]() {
    if constexpr (!kSplitKeys) {
#pragma unroll
      for (int rb = 0; rb < kBlocks; ++rb) {
        const float m_new = fmaxf(m_run[rb], m[rb]);
        const float f_run = merge_factor(m_run[rb], m_new), f = merge_factor(m[rb], m_new);
        m_run[rb] = m_new;
        l_run[rb] = fmaf(lsum[rb], f, l_run[rb] * f_run);
        if (__builtin_amdgcn_ballot_w64(f_run != 1.0f || f != 1.0f) == 0) {
#pragma unroll
          for (int d = 0; d < ND; ++d) o_run[rb][d] += o[rb][d];
        } else {
#pragma unroll
          for (int d = 0; d < ND; ++d) o_run[rb][d] = __builtin_elementwise_fma(o[rb][d], splat(f), o_run[rb][d] * f_run);
        }
        m[rb] = -INFINITY;
        lsum[rb] = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[rb][d] = splat(0.0f);
      }
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

  // where a pair's result goes: its partial, or its row of the output
  auto slot_of = [&](int p) -> int64_t {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (p >> lg);
    const int64_t at = tok * a.Hq + g * a.group + (p & (a.group - 1));
    return kSplitKeys ? at * a.n_seg + seg : at;
  };
  if constexpr (!kSplitKeys) fold();
#pragma unroll
  for (int rb = 0; rb < kBlocks; ++rb) {
    if (!row_ok[rb]) continue;
    const int64_t at = slot_of(pair0 + 32 * rb + lrow);
    if constexpr (kSplitKeys) {
      float* op = a.part_acc + at * D;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<float4*>(op + d * 32 + r4 * 8 + half * 4) =
              make_float4(o[rb][d][r4 * 4], o[rb][d][r4 * 4 + 1], o[rb][d][r4 * 4 + 2], o[rb][d][r4 * 4 + 3]);
      if (half == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(m[rb], lsum[rb]);
    } else {
      const float inv = 1.0f / l_run[rb];
      uint16_t* op = static_cast<uint16_t*>(a.out) + at * D;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          *reinterpret_cast<uint2*>(op + d * 32 + r4 * 8 + half * 4) =
              make_uint2(pack_bf16_rne(o_run[rb][d][r4 * 4] * inv, o_run[rb][d][r4 * 4 + 1] * inv),
                         pack_bf16_rne(o_run[rb][d][r4 * 4 + 2] * inv, o_run[rb][d][r4 * 4 + 3] * inv));
    }
  }
  // ---- the values that are not finite, to the rows that see them (a dimension per lane)
  __syncthreads();
  if (s_bad != 0 && !idle) {
    __builtin_amdgcn_s_waitcnt(0x0F70);
    const int pairs = min(32 * kBlocks, (len << lg) - pair0);
    for (int kt = kt_begin; kt < n_tiles; ++kt) {
      const int key0 = kt * kTileKeys;
      if (!(min(key0 + kTileKeys, n_hi) - 1 > tile_first || key0 < tile_mask_lo)) continue;
      for (int key = max(key0, wave_lo); key < min(key0 + kTileKeys, wave_last + 1); ++key) {
        const int32_t page = bt[key / kPage];
        const T* vr = vpool + (((int64_t)(page >= 0 && page < a.n_pages ? page : 0) * a.Hkv + g) * kPage + key % kPage) * D;
        for (int x = lane; x < D; x += 64) {
          const float v = load_value(vr + x);
          if (fabsf(v) < INFINITY) continue;
          for (int i = 0; i < pairs; ++i) {
            const int n = ctx + ((pair0 + i) >> lg);
            if (key > n || key < window_start(W, n + 1)) continue;
            const int64_t at = slot_of(pair0 + i);
            if constexpr (kSplitKeys)
              a.part_acc[at * D + x] = v;
            else
              static_cast<uint16_t*>(a.out)[at * D + x] = (uint16_t)(__float_as_uint(v) >> 16);
          }
        }
      }
    }
  }
}

// out = the rows' segments folded in ascending order, a wave per (layer, token, query head).
template <int D>
__global__ __launch_bounds__(256) void packed_fold_kernel(const PackedAttnArgs a) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= (int64_t)a.n_layers * a.seqs.n_tokens * a.Hq) return;
  const int64_t tok = id / a.Hq;
  const int l = (int)(tok / a.seqs.n_tokens), t = (int)(tok % a.seqs.n_tokens);
  const SeqUnit u = find_token(a.seqs, t);
  if (u.b < 0) return;
  const int n = u.range.ctx + u.at;
  const int s_lo = window_start(layer_window(a, l), n + 1) / kPackedSeg, s_hi = n / kPackedSeg;
  float m_run = -INFINITY, l_run = 0.0f, o_run[N] = {};
  for (int s = s_lo; s <= s_hi; ++s) {
    const int64_t at = id * a.n_seg + s;
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
    const float m_new = fmaxf(m_run, ml.x);
    const float f_run = merge_factor(m_run, m_new), f = merge_factor(ml.x, m_new);
    m_run = m_new;
    l_run = fmaf(ml.y, f, l_run * f_run);
#pragma unroll
    for (int x = 0; x < N; ++x) o_run[x] = fmaf(a.part_acc[at * D + lane * N + x], f, o_run[x] * f_run);
  }
  const float inv = 1.0f / l_run;
  uint16_t* op = static_cast<uint16_t*>(a.out) + id * D + lane * N;
#pragma unroll
  for (int x = 0; x < N; ++x) op[x] = __builtin_bit_cast(uint16_t, (__bf16)(o_run[x] * inv));
}

template <typename T, int D, int kBlocks>
hipError_t launch_d(const PackedAttnArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)packed_mfma_workgroups(a));
  if (a.n_seg > 1)
    packed_mfma_kernel<T, D, kBlocks, true><<<grid, 64 * kWaves, 0, stream>>>(a);
  else
    packed_mfma_kernel<T, D, kBlocks, false><<<grid, 64 * kWaves, 0, stream>>>(a);
  if (a.n_seg > 1)
    packed_fold_kernel<D><<<(unsigned)(((int64_t)a.n_layers * a.seqs.n_tokens * a.Hq + 3) / 4), 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const PackedAttnArgs& a, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_d<T, 64, 2>(a, stream);
    case 128: return launch_d<T, 128, 1>(a, stream);
    case 256: return launch_d<T, 256, 1>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

int packed_mfma_pairs(int D) { return 32 * kWaves * (D == 64 ? 2 : 1); }

hipError_t launch_packed_mfma(const PackedAttnArgs& a, int dtype, hipStream_t stream) {
  if (dtype == kDtypeBf16) return launch_t<uint16_t>(a, stream);
  if (dtype == kDtypeFp8) return launch_t<uint8_t>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace kvg
