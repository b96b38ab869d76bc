// Causal attention of packed sequences over a paged fp32 cache, on v_mfma_f32_32x32x2_f32: fp32 operands, products and sums.
//
// Workgroup = (layer, KV head, tile of 32 (row, query head) pairs of a sequence, heads fastest).  A segment of kPackedSeg
// keys (absolute multiples) is shared by the four waves, 128 keys each in blocks of 32 with an online softmax; the
// waves' states are folded in order through LDS, and the segments' after them: in registers, or, in a split
// launch (a workgroup per segment), by packed_fold_kernel with the same operations.  So a row's bytes do not
// depend on the launch.
//
//   S^T = K Q^T    C = 32 keys x 32 pairs; a lane's operand is one float of key (pair) lane % 32: step (j, e) takes dims
//                  8 j + e in lanes 0-31 and 8 j + 4 + e in lanes 32-63, so one 16-byte load feeds four steps; four
//                  accumulation chains, added pairwise
//   softmax        fp32, against the largest score so far
//   O^T += V^T P^T step r takes the keys of accumulator element r (8 (r / 4) + r % 4, lanes 32-63 four further), so P is the
//                  operand as it stands; block db of O^T is dims ND i + db of row i, so that a lane's ND values of a key
//                  are consecutive
//
// What bounds it: the matrix cores (64 cycles a step; the fp32 rate is a sixteenth of bf16's), with K and V from L2
// straight into registers several loads ahead; in small launches the walk of one workgroup.  Sixteen ragged chunks over 1k
// keys take 28 us at 4 / 2 heads x 64 (1.3 GFLOP) and the fold 5, and 507 us at 16 / 8 x 256 (41 TFLOP/s, where a large
// matrix product of the library reaches 154: one wave a SIMD, and half the pairs of a ragged tile are none).
#include "kvg_launch.h"
#include "kvg_packed_mfma.h"

#include <type_traits>

namespace kvg {

namespace {

constexpr int kWaves = 4;
constexpr int kWaveKeys = kPackedSeg / kWaves;

template <int N>
struct Floats {
  float x[N];
};
template <int N>
__device__ __forceinline__ Floats<N> load_floats(const float* p) {
  return *reinterpret_cast<const Floats<N>*>(p);
}

template <int D, bool kSplitKeys>
__global__ __launch_bounds__(64 * kWaves, 1) void packed_f32_kernel(const PackedAttnArgs a) {
  constexpr int NJ = D / 8;            // 16-byte K loads per block and lane
  constexpr int ND = D / 32;           // blocks of O^T
  constexpr int LK = 8, LV = D == 256 ? 4 : 8;        // K and V loads ahead
  constexpr int kChains = 4;           // accumulation chains of a score, one for each value of a load
  constexpr bool kQInLds = D == 256;   // the tile's queries, in registers where they fit
  constexpr int kPitch = 36;
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][32][kPitch];
  __shared__ float2 s_ml[kWaves][32];
  __shared__ int s_bad;
  __shared__ __attribute__((aligned(16))) Floats<4> s_q[kQInLds ? NJ : 1][64];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lrow = lane & 31, half = lane >> 5;
  const int lg = 31 - __builtin_clz(a.group);
  // (tile, layer, segment, KV head): see the bf16 tile kernel
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
  const SeqUnit u = find_unit(a.seqs, slot, [&](const SeqRange& s) { return (int)((((int64_t)s.len << lg) + 31) / 32); });
  if (u.b < 0) return;
  const SeqRange sq = u.range;
  const int pair0 = (u.count - 1 - u.at) * 32;
  const int W = layer_window(a, l);
  const int row = (pair0 + lrow) >> lg;
  const bool row_ok = row < sq.len;
  const int row_n = sq.ctx + row, row_lo = window_start(W, row_n + 1);
  const int first = sq.ctx + (pair0 >> lg), last = sq.ctx + min((pair0 + 31) >> lg, sq.len - 1);
  const int tile_lo = window_start(W, first + 1), mask_lo = window_start(W, last + 1);    // of the first row; keys all rows see start here
  const int tile_hi = last + 1;
  int seg_begin = tile_lo / kPackedSeg, seg_end = last / kPackedSeg + 1;
  if constexpr (kSplitKeys) {
    if (seg < seg_begin || seg >= seg_end) return;
    seg_begin = seg;
    seg_end = seg + 1;
  }
  const int64_t lbase = (int64_t)(a.layer0 + l) * a.layer_elems;
  const float* kpool = reinterpret_cast<const float*>(a.k_pool) + lbase;
  const float* vpool = reinterpret_cast<const float*>(a.v_pool) + lbase;
  const int32_t* bt = a.seqs.tables + (int64_t)u.b * a.seqs.max_pages;
  const int last_page = (tile_hi - 1) / kPage;

  Floats<4> q[kQInLds ? 1 : NJ];
  {
    const int p = pair0 + lrow;
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + (row_ok ? row : 0);
    const float* qp = static_cast<const float*>(a.q) + tok * a.q_stride + (int64_t)(g * a.group + (p & (a.group - 1))) * D + 4 * half;
    if constexpr (kQInLds) {
#pragma unroll
      for (int j = 0; j < NJ / kWaves; ++j) s_q[wave * (NJ / kWaves) + j][lane] = load_floats<4>(qp + 8 * (wave * (NJ / kWaves) + j));
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j) q[j] = load_floats<4>(qp + 8 * j);
    }
  }
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();

  // a thread's part of the folded result: pair t / 8, dims ND i + db of i = 4 (t % 8) + 0..3
  const int f_pair = threadIdx.x >> 3, f_i = (threadIdx.x & 7) * 4;
  float m_run = -INFINITY, l_run = 0.0f;
  float run[ND][4];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) run[d][e] = 0.0f;
  bool any_bad = false;

  for (int s_id = seg_begin; s_id < seg_end; ++s_id) {
    // ---- this wave's blocks
    const int key_end = min(s_id * kPackedSeg + (wave + 1) * kWaveKeys, tile_hi);
    const int key_begin = max(s_id * kPackedSeg + wave * kWaveKeys, tile_lo & ~31);
    const int n_blocks = key_end > key_begin ? (key_end - key_begin + 31) / 32 : 0;
    const int32_t pg = bt[min(key_begin / kPage + (lane & 15), last_page)];        // the wave's pages (8), one per lane
    auto page_row = [&](int page_slot) -> int64_t {                                // first row of the (page, head) slab
      int32_t page = __builtin_amdgcn_readlane(pg, min(page_slot, 15));
      page = (page >= 0 && page < a.n_pages) ? page : 0;
      return ((int64_t)page * a.Hkv + g) * kPage;
    };
    auto k_ptr = [&](int i) -> const float* {
      const int64_t ra = page_row(2 * i), rb = page_row(2 * i + 1);
      return kpool + ((lrow < kPage ? ra : rb) + lrow % kPage) * D + 4 * half;
    };
    f32x16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = splat(0.0f);
    float m = -INFINITY, lsum = 0.0f;
    Floats<4> kf[LK];
    const float* kp = n_blocks > 0 ? k_ptr(0) : kpool;
    if (n_blocks > 0) {
#pragma unroll
      for (int j = 0; j < LK; ++j) kf[j] = load_floats<4>(kp + 8 * j);
    }
    for (int i = 0; i < n_blocks; ++i) {
      const int kb = key_begin + 32 * i;
      int q_lane = lane;
      asm volatile("" : "+v"(q_lane));       // the queries are read from LDS in every block, not once into registers
      auto query = [&](int j) -> Floats<4> { return kQInLds ? s_q[j][q_lane] : q[kQInLds ? 0 : j]; };
      const float* kp_next = k_ptr(min(i + 1, n_blocks - 1));
      const float* vp0 = vpool + (page_row(2 * i) + 4 * half) * D + ND * lrow;
      const float* vp1 = vpool + (page_row(2 * i + 1) + 4 * half) * D + ND * lrow;
      Floats<ND> vf[LV];
      auto vfetch = [&](int r) { vf[r % LV] = load_floats<ND>((r < 8 ? vp0 : vp1) + (8 * ((r / 4) & 1) + r % 4) * D); };
#pragma unroll
      for (int r = 0; r < LV; ++r) vfetch(r);
      f32x16 c[kChains];
#pragma unroll
      for (int x = 0; x < kChains; ++x) c[x] = splat(0.0f);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const Floats<4> k = kf[j % LK], qj = query(j);
        kf[j % LK] = load_floats<4>((j + LK < NJ ? kp : kp_next) + 8 * ((j + LK) % NJ));
#pragma unroll
        for (int e = 0; e < kChains; ++e) c[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x[e], qj.x[e], c[e], 0, 0, 0);
      }
      kp = kp_next;
      f32x16 s = (c[0] + c[1]) + (c[2] + c[3]);
      const bool edge = kb + 31 > first || kb < mask_lo;       // keys that some row does not see
      if (edge) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t key = kb + half * 4 - row_lo + (r >> 2) * 8 + (r & 3);
          s[r] = key <= (uint32_t)(row_n - row_lo) ? s[r] : -INFINITY;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
      const float2 mh = halves32(mx);
      const float m_new = fmaxf(m, fmaxf(mh.x, mh.y) * a.scale_log2);
      const bool raised = m_new > m;
      const float alpha = raised ? __builtin_amdgcn_exp2f(m - m_new) : 1.0f;
      m = m_new;
      const float m_ref = m == -INFINITY ? 0.0f : m;           // no key seen yet: every weight is 0
      float psum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -m_ref));
        psum += s[r];
      }
      const float2 ph = halves32(psum);
      lsum = fmaf(lsum, alpha, ph.x + ph.y);
      if (__builtin_amdgcn_ballot_w64(raised) != 0) {
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= alpha;
      }
      // a masked key weighs 0, and 0 times an Inf or NaN among its values would reach rows that do not see it: in blocks with
      // such keys the products take the finite values, and the others are given to the rows that see them at the end
      auto pv = [&](auto masked) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          Floats<ND> v = vf[r % LV];
          if (r + LV < 16) vfetch(r + LV);
          if constexpr (decltype(masked)::value) {
            const int key = kb + half * 4 + (r >> 2) * 8 + (r & 3);
#pragma unroll
            for (int d = 0; d < ND; ++d) {
              const bool finite = fabsf(v.x[d]) < INFINITY;
              any_bad = any_bad || (!finite && key < tile_hi);
              v.x[d] = finite ? v.x[d] : 0.0f;
            }
          }
#pragma unroll
          for (int d = 0; d < ND; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.x[d], s[r], o[d], 0, 0, 0);
        }
      };
      if (edge || kb + 32 > tile_hi)
        pv(std::true_type{});
      else
        pv(std::false_type{});
    }
    // ---- the four waves' states in order, after the segments before
    if (half == 0) s_ml[wave][lrow] = make_float2(m, lsum);
    FoldFactors f[kWaves];
    float m_seg = -INFINITY, l_seg = 0.0f;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<float4*>(&s_o[wave][lrow][8 * r4 + 4 * half]) = make_float4(o[d][4 * r4], o[d][4 * r4 + 1], o[d][4 * r4 + 2], o[d][4 * r4 + 3]);
      __syncthreads();
      FoldFactors fs = {0.0f, 0.0f};
      if (d == 0) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float2 ml = s_ml[w][f_pair];
          f[w] = fold_factors(m_seg, l_seg, ml.x, ml.y);
        }
      }
      float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(&s_o[w][f_pair][f_i]);
        const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[e], f[w].part, acc[e] * f[w].run);
      }
      __syncthreads();
      if constexpr (kSplitKeys) {
#pragma unroll
        for (int e = 0; e < 4; ++e) run[d][e] = acc[e];
      } else {
        // the segment's state into the running one: factors from the references before and after
        const float m_new = fmaxf(m_run, m_seg);
        fs = {merge_factor(m_run, m_new), merge_factor(m_seg, m_new)};
#pragma unroll
        for (int e = 0; e < 4; ++e) run[d][e] = fmaf(acc[e], fs.part, run[d][e] * fs.run);
      }
    }
    if constexpr (kSplitKeys) {
      m_run = m_seg;
      l_run = l_seg;
    } else {
      fold_factors(m_run, l_run, m_seg, l_seg);
    }
  }

  // ---- the partial, or the result
  const int64_t block = part_block(a, a.part.n_seg, l, slot, g, 1, 0, seg);
  auto row_of = [&](int p) -> int64_t {
    const int64_t tok = (int64_t)l * a.seqs.n_tokens + sq.row0 + ((pair0 + p) >> lg);
    return tok * a.Hq + g * a.group + ((pair0 + p) & (a.group - 1));
  };
  const int pairs = min(32, (sq.len << lg) - pair0);
  if (f_pair < pairs) {
    const float inv = kSplitKeys ? 1.0f : 1.0f / l_run;
#pragma unroll
    for (int j = 0; j < ND; ++j) {            // dims ND f_i + 4 j + 0..3
      Floats<4> v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v.x[i] = kSplitKeys ? run[(4 * j + i) % ND][(4 * j + i) / ND] : row_result(run[(4 * j + i) % ND][(4 * j + i) / ND], inv);
      const int x = ND * f_i + 4 * j;
      float* dst = kSplitKeys ? a.part.acc + block * (32 * D) + part_at(f_pair, x) : static_cast<float*>(a.out) + row_of(f_pair) * D + x;
      *reinterpret_cast<Floats<4>*>(dst) = v;
    }
    if (kSplitKeys && (threadIdx.x & 7) == 0) *reinterpret_cast<float2*>(a.part.ml + (block * 32 + f_pair) * 2) = make_float2(m_run, l_run);
  }
  if (__builtin_amdgcn_ballot_w64(any_bad) != 0) s_bad = 1;
  __syncthreads();
  if (s_bad != 0) {
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    if (wave != 0) return;
    put_bad_values(a, vpool, bt, g, max(seg_begin * kPackedSeg, tile_lo), min(seg_end * kPackedSeg, tile_hi), W, sq.ctx, lg, pair0, pairs,
                   [&](int p, int x, float v) {
                     float* to = kSplitKeys ? a.part.acc + block * (32 * D) + part_at(p, x) : static_cast<float*>(a.out) + row_of(p) * D + x;
                     *to = take_in(*to, v);
                   });
  }
}

template <int D>
hipError_t launch_f32_d(const PackedAttnArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)packed_tile_workgroups(a);
  if (a.part.n_seg > 1)
    packed_f32_kernel<D, true><<<grid, 64 * kWaves, 0, stream>>>(a);
  else
    packed_f32_kernel<D, false><<<grid, 64 * kWaves, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_f32(const PackedAttnArgs& a, hipStream_t stream) {
  switch (a.D) {
    case 64: return launch_f32_d<64>(a, stream);
    case 128: return launch_f32_d<128>(a, stream);
    case 256: return launch_f32_d<256>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace kvg
