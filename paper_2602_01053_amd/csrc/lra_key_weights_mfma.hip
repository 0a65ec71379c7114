// Attention weight per cached token on the matrix cores (bf16 caches with one L): lra_key_weights of the header.
//
//   Qt    = Q B_K^T, as two bf16 terms (16 bits of mantissa: the second is what the first left over)
//   stats: per query row and key share  m = max s, l = sum exp2(s - m),  s = scale log2(e) (K_base Q^T + L Qt^T)
//   lse   = m + log2 l over the shares
//   sums:  w[j] = decay w[j] + sum over rows exp2(s_j - lse)
//
// Scores are products of bf16 in fp32, so the weights come out as exactly as fp32 sums of them allow; Qt rounded to one
// bf16 term alone would put 1e-3 into each.  K is read twice, since a weight needs its row's maximum and sum first.
//
// K comes through LDS (buffer_load ... lds, swizzled as in the prefill kernels) past query rows held 32 to a wave.  In the
// statistics a workgroup owns 128 rows of a sequence and a share of its keys, 64 at a time; in the sums it owns keys and walks
// the kv heads and the rows, so that the sum over them stays in the
// workgroup, is added up in one fixed order, and needs no atomics.  (K rows straight to registers as matrix operands: 64
// lanes of a load then touch 64 places, which held the batch of 16 sequences to 3.0 and 2.3 TB/s.)
#include "lra_decode_util.h"
#include "lra_key_weights.h"
#include "lra_prefill_util.h"

namespace lra {

template <int N>
__device__ __forceinline__ float lane_ror(float v) {  // rotation inside each row of sixteen lanes
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
}

// The 64-key tiles of one sequence, requested by the four waves of a workgroup.  Tokens that no query of the sequence sees
// (cut_lo to cut_hi - 1) and those past the end read as zeros and touch no memory; their blocks may have any id.
template <int D, int RP, bool PAGED>
struct KeyTiles {
  static constexpr int KCH = D / 8, KROWS = 64 / KCH, LCH = RP / 8, LROWS = 64 / LCH;
  static constexpr int K_BYTES = 64 * D * 2, L_BYTES = 64 * RP * 2;
  const WeightsParams& p;
  int t, n_t, cut_lo, cut_hi, wave, lane;
  uint32_t lds0, ts2, lp2, k_voff, ids[4];
  pf_u32x4 rs_l;
  __device__ __forceinline__ bool kept(int tok) const { return tok < n_t && (tok < cut_lo || tok >= cut_hi); }
  __device__ __forceinline__ KeyTiles(const WeightsParams& p_, unsigned char* smem, int t_, int n_t_, int cut_lo_, int cut_hi_, int wave_, int lane_)
      : p(p_), t(t_), n_t(n_t_), cut_lo(cut_lo_), cut_hi(cut_hi_), wave(wave_), lane(lane_) {
    lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem)));
    ts2 = static_cast<uint32_t>(p.kv_token_stride) * 2u;
    lp2 = static_cast<uint32_t>(p.l_row_stride) * 2u;
    k_voff = static_cast<uint32_t>(lane / KCH) * ts2 + ((lane % KCH ^ pf_swz_k<D>(wave * KROWS + lane / KCH)) << 4);
    const uint32_t l_rows = PAGED ? static_cast<uint32_t>(p.num_blocks) * 16u : static_cast<uint32_t>(n_t);
    rs_l = pf_rsrc(p.l, (l_rows - 1u) * lp2 + static_cast<uint32_t>(p.rank) * 2u);
    ids[0] = ids[1] = ids[2] = ids[3] = 0u;
  }
  // block ids of the tile at key j
  __device__ __forceinline__ void look_up(int j) {
    if constexpr (PAGED) {
      const int last = (n_t - 1) >> 4;
#pragma unroll
      for (int b = 0; b < 4; ++b)
        ids[b] = static_cast<uint32_t>(PF_CONST_I32(p.block_table)[static_cast<int64_t>(t) * p.max_blocks_per_seq + min((j >> 4) + b, last)]);
    }
  }
  // this wave's share of K's rows of head h to LDS at byte `at`
  __device__ __forceinline__ void issue_k(int j, int h, uint32_t at) const {
#pragma unroll
    for (int q = 0; q < 64 / KROWS / 4; ++q) {
      const int i = wave + 4 * q, tok = j + i * KROWS;  // (the rows of one load lie in one block, the swizzle does not depend on q)
      const bool any = tok < n_t && (tok < cut_lo || min(tok + KROWS, n_t) > cut_hi);
      const int nv = any ? min(KROWS, n_t - tok) : 0;
      const uint32_t bytes = nv > 0 ? static_cast<uint32_t>(nv - 1) * ts2 + D * 2 : 0u;
      const uint32_t blk = D == 128 ? ids[q] : (wave < 2 ? ids[2 * q] : ids[(2 * q + 1) & 3]);  // (block (i KROWS) / 16 of the tile)
      const int64_t off = static_cast<int64_t>(h) * p.kv_head_stride +
                          (PAGED ? static_cast<int64_t>(blk) * p.kv_block_stride + static_cast<int64_t>(tok & 15) * p.kv_token_stride
                                 : static_cast<int64_t>(tok) * p.kv_token_stride);
      pf_load16_to_lds(pf_rsrc(static_cast<const bf16_t*>(p.k_base) + off, bytes), lds0 + at + i * 1024, kept(tok + lane / KCH) ? k_voff : kPfOob, 0);
    }
  }
  __device__ __forceinline__ void issue_l(int j, uint32_t at) const {
#pragma unroll
    for (int q = 0; q < (LCH + 3) / 4; ++q) {
      const int i = wave + 4 * q;
      if (i < LCH) {
        const int row = i * LROWS + lane / LCH, tok = j + row;
        uint32_t index = static_cast<uint32_t>(tok);
        if constexpr (PAGED) {
          const int b = row >> 4;
          const uint32_t lo2 = b == 0 ? ids[0] : ids[1], hi2 = b == 2 ? ids[2] : ids[3];
          index = (b < 2 ? lo2 : hi2) * 16u + (static_cast<uint32_t>(tok) & 15u);
        }
        const int ch = lane % LCH ^ pf_swz_l<LCH>(row);
        pf_load16_to_lds(rs_l, lds0 + at + i * 1024, kept(tok) && ch * 8 < p.rank ? index * lp2 + (ch << 4) : kPfOob, 0);
      }
    }
  }
};

// Scores of a tile's 64 keys and a wave's 32 rows: s[kt][i] is key 32 kt + 8 (i / 4) + 4 g2 + i % 4 of row l32, minus infinity
// where it is not seen (pos: the row's position, pos_first and pos_last the wave's).
template <int D, int RP, bool HAS_BK>
__device__ __forceinline__ void tile_scores(const WeightsParams& p, const unsigned char* k_lds, const unsigned char* l_lds, int l32, int g2,
                                            const pf_bf16x8 (&q)[D / 16], const pf_bf16x8 (&hi)[RP / 16], const pf_bf16x8 (&lo)[RP / 16], int j,
                                            int pos, int pos_first, int pos_last, pf_f32x16 (&s)[2]) {
  constexpr int KS = D / 16, RKS = RP / 16, LCH = RP / 8;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
  if constexpr (HAS_BK) {
#pragma unroll
    for (int ks = 0; ks < RKS; ++ks) {
      pf_bf16x8 a[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const unsigned char* row = l_lds + (32 * kt + l32) * (RP * 2) + g2 * 8;
        const uint2 x = *reinterpret_cast<const uint2*>(row + (((2 * ks) ^ pf_swz_l<LCH>(l32)) << 4));
        const uint2 y = *reinterpret_cast<const uint2*>(row + (((2 * ks + 1) ^ pf_swz_l<LCH>(l32)) << 4));
        a[kt] = pf_as_bf16x8(make_uint4(x.x, x.y, y.x, y.y));
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[kt], lo[ks], s[kt], 0, 0, 0);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[kt], hi[ks], s[kt], 0, 0, 0);
    }
  }
  const int k_pre = l32 * (D * 2) + (pf_swz_k<D>(l32) << 4);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint4 a = *reinterpret_cast<const uint4*>(k_lds + (k_pre ^ ((2 * ks + g2) << 4)) + kt * 32 * D * 2);
      s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(a), q[ks], s[kt], 0, 0, 0);
    }
  if (j + 63 > pos_first) {  // some row does not see the last key
    const int last = pos - j - 4 * g2;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * kt + 8 * (i >> 2) + (i & 3) > last) s[kt][i] = -INFINITY;
  }
  if (p.window > 0 && j + p.window <= pos_last && j + 64 > p.sinks) {  // some row's window starts behind the first key
    const int from = p.sinks - j - 4 * g2;  // hidden: `hidden` keys from here on
    const uint32_t hidden = static_cast<uint32_t>(max(0, pos - p.window + 1 - p.sinks));
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (static_cast<uint32_t>(32 * kt + 8 * (i >> 2) + (i & 3) - from) < hidden) s[kt][i] = -INFINITY;
  }
}

// (query of the sequence, q head of the group) of row `at` of a sequence's rows
__device__ __forceinline__ void split_row(int at, int group, int& tok, int& g) {
  tok = at / group;
  g = at - tok * group;
}

template <int D, int RP, bool HAS_BK, bool PAGED>
__global__ __launch_bounds__(256, 2) void weights_stats_mfma_kernel(WeightsParams p) {
  typedef KeyTiles<D, RP, PAGED> Tiles;
  constexpr int KS = D / 16, RKS = RP / 16, RB = (RP + 31) / 32;
  constexpr int STAGE = Tiles::K_BYTES + (HAS_BK ? Tiles::L_BYTES : 0);
  __shared__ __align__(16) unsigned char smem[2 * STAGE];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = p.group, Hkv = p.n_kv_heads;
  // (kv head fastest: with eight of them an XCD takes the workgroups of one)
  const int rest = blockIdx.x / Hkv, h = blockIdx.x - rest * Hkv;
  const int place = rest / p.n_splits, split = rest - place * p.n_splits;
  const BatchTiles item = batch_tiles(p, place, lane);
  const int n_rows = item.n_queries * G;
  if (static_cast<int64_t>(item.tile) * 128 >= n_rows) return;
  const int q0 = item.tile * 128, step = p.causal ? 1 : 0, n_t = item.n_t;
  const bool live = q0 + wave * 32 < n_rows;
  int tok, g;  // of this lane's row (the last one again past the end)
  split_row(min(q0 + wave * 32 + l32, n_rows - 1), G, tok, g);
  const int row = (item.first_query + tok) * G + g;
  const int pos = item.first_pos + step * tok;
  const int pos_first = __builtin_amdgcn_readfirstlane(pos), pos_last = __builtin_amdgcn_readlane(pos, 31);
  const int wg_first = item.first_pos + step * (q0 / G), wg_last = item.first_pos + step * ((min(q0 + 128, n_rows) - 1) / G);
  const int lo = p.window > 0 ? max(0, wg_first - p.window + 1) : 0, sinks = min(p.sinks, lo);
  const int sink_tiles = (sinks + 63) / 64, gap = max(0, lo / 64 - sink_tiles);
  const int n_tiles = wg_last < 0 ? 0 : wg_last / 64 + 1 - gap;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / p.n_splits);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / p.n_splits);
  auto key_of = [&](int tile) __attribute__((always_inline)) -> int { return (tile < sink_tiles ? tile : tile + gap) * 64; };
  float* out = p.stats + ((static_cast<int64_t>(h) * p.n_splits + split) * p.rows_per_head + row) * 2;
  const bool mine = live && q0 + wave * 32 + l32 < n_rows && g2 == 0;
  if (t0 >= t1 && split > 0) {  // (share 0 leaves Qt whatever it has to do)
    if (mine) *reinterpret_cast<float2*>(out) = make_float2(-INFINITY, 0.f);
    return;
  }
  Tiles tiles(p, smem, item.t, max(n_t, 1), sinks, lo, wave, lane);
  if (t0 < t1) {
    tiles.look_up(key_of(t0));
    tiles.issue_k(key_of(t0), h, 0);
    if (HAS_BK) tiles.issue_l(key_of(t0), Tiles::K_BYTES);
    if (t0 + 1 < t1) tiles.look_up(key_of(t0 + 1));
  }
  pf_bf16x8 q[KS], hi[RKS], low[RKS];
  {
    const bf16_t* qr = static_cast<const bf16_t*>(p.q) + (static_cast<int64_t>(item.first_query + tok) * p.n_q_heads + h * G + g) * D + g2 * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qr + ks * 16));
  }
#pragma unroll
  for (int ks = 0; ks < RKS; ++ks) hi[ks] = low[ks] = pf_as_bf16x8(make_uint4(0u, 0u, 0u, 0u));
  if constexpr (HAS_BK) {
    // Qt^T = B_K Q^T, one product per adapter of the wave's rows (batch_tiles_body has the same with one bf16 term): element e
    // of k-step ks is rank 16 ks + 8 (e / 4) + 4 g2 + e % 4, the order in which the L operand is read
    const int64_t ldb = static_cast<int64_t>(Hkv) * D;
    const bf16_t* bk = static_cast<const bf16_t*>(p.b_k) + h * D;
    const int tok_a = __builtin_amdgcn_readfirstlane(tok), tok_b = __builtin_amdgcn_readlane(tok, 31);
    const int n_it = !live ? 0 : (p.causal ? 1 : tok_b - tok_a + 1);
    pf_u32x4 x[RB][KS];
    auto request = [&](int it) __attribute__((always_inline)) {
      const int a = p.causal ? item.adapter : min(max(__builtin_amdgcn_readfirstlane(p.query_adapter[item.first_query + tok_a + it]), 0), p.n_adapters - 1);
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(bk) + static_cast<int64_t>(a) * p.rank * ldb, 0,
                                                                          static_cast<int>((static_cast<int64_t>(p.rank - 1) * ldb + D) * 2), 0x00020000);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int rho = b * 32 + l32;
        const uint32_t off = rho < p.rank ? static_cast<uint32_t>(rho * ldb * 2 + g2 * 16) : kPfOob;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) x[b][ks] = __builtin_amdgcn_raw_buffer_load_b128(rs, off, ks * 32, 0);
      }
    };
    if (n_it > 0) request(0);
#pragma unroll 1
    for (int it = 0; it < n_it; ++it) {
      pf_f32x16 acc[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pf_bf16x8, x[b][ks]), q[ks], acc[b], 0, 0, 0);
      }
      if (it + 1 < n_it) request(it + 1);
      if (p.causal || tok == tok_a + it) {
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks) {
          uint32_t w[2][4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x0 = acc[ks >> 1][(ks & 1) * 8 + 2 * e], x1 = acc[ks >> 1][(ks & 1) * 8 + 2 * e + 1];
            w[0][e] = pf_pack2(x0, x1);
            const float r0 = x0 - __uint_as_float(w[0][e] << 16), r1 = x1 - __uint_as_float(w[0][e] & 0xffff0000u);
            w[1][e] = pf_pack2(__builtin_isfinite(r0) ? r0 : 0.f, __builtin_isfinite(r1) ? r1 : 0.f);
          }
          hi[ks] = pf_as_bf16x8(make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]));
          low[ks] = pf_as_bf16x8(make_uint4(w[1][0], w[1][1], w[1][2], w[1][3]));
        }
      }
    }
    if (split == 0 && live) {  // for the sums (rows past the end write the last one's again)
      bf16_t* qt = reinterpret_cast<bf16_t*>(p.qt) + (static_cast<int64_t>(h) * p.rows_per_head + row) * 2 * RP + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < RKS; ++ks) {
        *reinterpret_cast<pf_u32x4*>(qt + ks * 16) = __builtin_bit_cast(pf_u32x4, hi[ks]);
        *reinterpret_cast<pf_u32x4*>(qt + RP + ks * 16) = __builtin_bit_cast(pf_u32x4, low[ks]);
      }
    }
  }
  float m = -INFINITY, l = 0.f;
  const float sc = p.scale * 1.44269504088896340736f;
  for (int tile = t0; tile < t1; ++tile) {
    const uint32_t at = ((tile - t0) & 1) * STAGE;
    pf_wait_vm0();
    __syncthreads();  // this tile is here for everyone, and everyone is done with the one before
    if (tile + 1 < t1) {
      tiles.issue_k(key_of(tile + 1), h, at ^ STAGE);
      if (HAS_BK) tiles.issue_l(key_of(tile + 1), (at ^ STAGE) + Tiles::K_BYTES);
      if (tile + 2 < t1) tiles.look_up(key_of(tile + 2));
    }
    const int j = key_of(tile);
    if (!live || j > pos_last || (p.window > 0 && j + 63 + p.window <= pos_first && j >= p.sinks)) continue;
    pf_f32x16 s[2];
    tile_scores<D, RP, HAS_BK>(p, smem + at, smem + at + Tiles::K_BYTES, l32, g2, q, hi, low, j, pos, pos_first, pos_last, s);
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
    const float m_new = fmaxf(m, tile_reference(mx * sc));
    const float nm = m_new == -INFINITY ? 0.f : -m_new;
    float sum = l * __builtin_amdgcn_exp2f(m + nm);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, nm));
    l = sum;
    m = m_new;
  }
  const float m2 = pf_partner32(m), l2 = pf_partner32(l);
  const float top = fmaxf(m, m2), nt = top == -INFINITY ? 0.f : -top;
  if (mine) *reinterpret_cast<float2*>(out) = make_float2(top, l * __builtin_amdgcn_exp2f(m + nt) + l2 * __builtin_amdgcn_exp2f(m2 + nt));
}

// lse of rows by four threads each (many rows; where a sequence has 32 at most the sums do it themselves)
__global__ __launch_bounds__(256) void weights_lse_kernel(WeightsParams p) {
  __shared__ float2 part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y;
  const int row = min(static_cast<int>(blockIdx.x) * 64 + lane, p.rows_per_head - 1);
  const float2* ml = reinterpret_cast<const float2*>(p.stats) + static_cast<int64_t>(h) * p.n_splits * p.rows_per_head + row;
  float2 x[8];  // (at most 32 shares)
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = ml[static_cast<int64_t>(min(wave + 4 * i, p.n_splits - 1)) * p.rows_per_head];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (wave + 4 * i < p.n_splits) m = fmaxf(m, x[i].x);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (wave + 4 * i < p.n_splits) l = fmaf(x[i].y, __builtin_amdgcn_exp2f(x[i].x - (m == -INFINITY ? 0.f : m)), l);
  part[wave][lane] = make_float2(m, l);
  __syncthreads();
  if (wave != 0 || static_cast<int>(blockIdx.x) * 64 + lane >= p.rows_per_head) return;
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w][lane].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) sum = fmaf(part[w][lane].y, __builtin_amdgcn_exp2f(part[w][lane].x - (top == -INFINITY ? 0.f : top)), sum);
  p.lse[static_cast<int64_t>(h) * p.rows_per_head + row] = sum == 0.f ? INFINITY : top + log2f(sum);
}

// Many rows: a workgroup owns 128 keys, 32 to a wave, which holds a head's K rows of them as matrix operands while Q walks through
// LDS 64 rows at a time, read by all four waves.  Short or few sequences have too few workgroups for the chip: then the heads
// are divided too, and weights_join_kernel adds the groups' sums in their order.  64 queries of 18 k tokens, 8 kv heads, d = 128:
// 29 us and the join's 4.7 (with 64 keys to a workgroup, 128 rows at a time past K in LDS: 45); instruction issue and the turn
// of a step, 64 rows, bound it.
constexpr int kSumKeys = 128;
template <int D, int RP, bool HAS_BK, bool PAGED>
__global__ __launch_bounds__(256, 2) void weights_sum_mfma_kernel(WeightsParams p) {
  typedef KeyTiles<D, RP, PAGED> Tiles;
  constexpr int KS = D / 16, RKS = RP / 16, KCH = D / 8, KROWS = 64 / KCH, LCH = RP / 8, Q_BYTES = 64 * D * 2;
  constexpr bool QT_EARLY = RP < 64;  // (64 registers of it would send d = 128 to scratch memory)
  constexpr int L_AT = 2 * Tiles::K_BYTES, Q_AT = L_AT + (HAS_BK ? 2 * Tiles::L_BYTES : 0);
  __shared__ __align__(16) unsigned char smem[Q_AT + 2 * Q_BYTES];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j0 = blockIdx.x * kSumKeys, t = blockIdx.y, G = p.group;
  const int n_t = min(PF_CONST_I32(p.seq_lens)[t], p.max_seq_len);
  if (j0 >= n_t) return;
  const int c0 = t > 0 ? min(max(PF_CONST_I32(p.seq_query_start)[t], 0), p.n_queries) : 0;
  const int c1 = t + 1 < p.n_seqs ? min(max(PF_CONST_I32(p.seq_query_start)[t + 1], c0), p.n_queries) : p.n_queries;
  const int n_rows = (c1 - c0) * G, step = p.causal ? 1 : 0;
  const int first_pos = p.causal ? n_t - (c1 - c0) : n_t - 1;
  const int lo = p.window > 0 ? max(0, first_pos - p.window + 1) : 0, sinks = min(p.sinks, lo);
  const float sc = p.scale * 1.44269504088896340736f;
  pf_f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  if (n_rows > 0 && (j0 < sinks || j0 + kSumKeys > lo)) {
    Tiles tile_a(p, smem, t, n_t, sinks, lo, wave, lane), tile_b = tile_a;
    tile_a.look_up(j0);
    tile_b.look_up(j0 + 64);
    int h = p.n_kv_heads * static_cast<int>(blockIdx.z) / static_cast<int>(gridDim.z);
    const int h_end = p.n_kv_heads * (static_cast<int>(blockIdx.z) + 1) / static_cast<int>(gridDim.z);
    auto request_k = [&](int head) __attribute__((always_inline)) {
      tile_a.issue_k(j0, head, 0);
      tile_b.issue_k(j0 + 64, head, Tiles::K_BYTES);
    };
    auto request_q = [&](int head, int rg, uint32_t at) __attribute__((always_inline)) {
      const int r0 = rg * 64;
      int tok0, head0;
      split_row(r0, G, tok0, head0);
      const pf_u32x4 rs = pf_rsrc(static_cast<const bf16_t*>(p.q) + (static_cast<int64_t>(c0 + tok0) * p.n_q_heads + head * G) * D, 0x7ffff000u);
#pragma unroll
      for (int i = 0; i < 64 / KROWS / 4; ++i) {
        // (past the end the last row again: zeros would turn infinite keys into NaN)
        const int r = (wave + 4 * i) * KROWS + lane / KCH, in = head0 + min(r, n_rows - 1 - r0), dt = (in * p.row_mul) >> 16;
        const uint32_t off = static_cast<uint32_t>((dt * p.n_q_heads + in - dt * G) * D * 2) + ((lane % KCH ^ pf_swz_k<D>(r)) << 4);
        pf_load16_to_lds(rs, tile_a.lds0 + at + (wave + 4 * i) * 1024, off, 0);
      }
    };
    const int rgs = (n_rows + 63) / 64;
    if (HAS_BK) {
      tile_a.issue_l(j0, L_AT);
      tile_b.issue_l(j0 + 64, L_AT + Tiles::L_BYTES);
    }
    request_k(h);
    request_q(h, 0, Q_AT);
    const int jw = j0 + 32 * wave;  // the wave's first key
    pf_bf16x8 ka[KS], la[RKS];
    uint32_t q_at = Q_AT;
    const int pre = l32 * (D * 2) + (pf_swz_k<D>(l32) << 4);
    bool first = true;
    for (; h < h_end; ++h) {
      const bf16_t* qt_h = reinterpret_cast<const bf16_t*>(p.qt) + (static_cast<int64_t>(h) * p.rows_per_head + static_cast<int64_t>(c0) * G) * 2 * RP + g2 * 8;
      const float* lse_h = p.lse + static_cast<int64_t>(h) * p.rows_per_head + static_cast<int64_t>(c0) * G;
      for (int rg = 0; rg < rgs; ++rg) {
        pf_wait_vm0();
        lds_fence();
        __syncthreads();  // these rows (and K of the head) are here for everyone, and everyone is done with the rows before
        if (rg == 0) {
          const unsigned char* k = smem + wave * 32 * D * 2;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) ka[ks] = pf_as_bf16x8(*reinterpret_cast<const uint4*>(k + (pre ^ ((2 * ks + g2) << 4))));
          if (HAS_BK && first) {
            const unsigned char* row = smem + L_AT + (32 * wave + l32) * (RP * 2) + g2 * 8;
#pragma unroll
            for (int ks = 0; ks < RKS; ++ks) {
              const uint2 x = *reinterpret_cast<const uint2*>(row + (((2 * ks) ^ pf_swz_l<LCH>(l32)) << 4));
              const uint2 y = *reinterpret_cast<const uint2*>(row + (((2 * ks + 1) ^ pf_swz_l<LCH>(l32)) << 4));
              la[ks] = pf_as_bf16x8(make_uint4(x.x, x.y, y.x, y.y));
            }
          }
          first = false;
          if (h + 1 < h_end) {
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): a wave reads only K rows that
            __syncthreads();                     // others requested: all have read theirs before the next head's come
            request_k(h + 1);
          }
        }
        const int r0 = rg * 64;
        // lse and Qt of this lane's two rows: on the way while K Q^T is formed
        float nl[2];
        pf_u32x4 hi[2][RKS], low[2][RKS];
        auto load_qt = [&](int rt, int r) __attribute__((always_inline)) {
          const bf16_t* row = qt_h + static_cast<int64_t>(r) * 2 * RP;
#pragma unroll
          for (int ks = 0; ks < RKS; ++ks) {
            hi[rt][ks] = *reinterpret_cast<const pf_u32x4*>(row + ks * 16);
            low[rt][ks] = *reinterpret_cast<const pf_u32x4*>(row + RP + ks * 16);
          }
        };
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
          const int r = min(r0 + 32 * rt + l32, n_rows - 1);
          nl[rt] = lse_h[r];
          if constexpr (HAS_BK && QT_EARLY) load_qt(rt, r);
        }
        const int pos_first = first_pos + step * __builtin_amdgcn_readfirstlane(r0 / G);
        const int pos_last = first_pos + step * __builtin_amdgcn_readfirstlane(min(r0 + 63, n_rows - 1) / G);
        const bool live = jw <= pos_last && !(p.window > 0 && jw + 31 + p.window <= pos_first && jw >= p.sinks);
        pf_f32x16 s[2];
        if (live) {
#pragma unroll
          for (int rt = 0; rt < 2; ++rt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[rt][i] = 0.f;
          // (two k-steps of Q read ahead of the products: left to itself the compiler waits for each read)
          uint4 q[2][2][2];
          auto read_q = [&](int part) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int rt = 0; rt < 2; ++rt)
                q[part & 1][k][rt] = *reinterpret_cast<const uint4*>(smem + q_at + (pre ^ ((2 * (2 * part + k) + g2) << 4)) + rt * 32 * D * 2);
          };
          read_q(0);
#pragma unroll
          for (int part = 0; part < KS / 2; ++part) {
            if (part + 1 < KS / 2) read_q(part + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int rt = 0; rt < 2; ++rt)
                s[rt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[2 * part + k], pf_as_bf16x8(q[part & 1][k][rt]), s[rt], 0, 0, 0);
          }
          if constexpr (HAS_BK && !QT_EARLY) {
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) load_qt(rt, min(r0 + 32 * rt + l32, n_rows - 1));
          }
          if constexpr (HAS_BK) {
#pragma unroll
            for (int ks = 0; ks < RKS; ++ks)
#pragma unroll
              for (int rt = 0; rt < 2; ++rt) {
                s[rt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(la[ks], __builtin_bit_cast(pf_bf16x8, low[rt][ks]), s[rt], 0, 0, 0);
                s[rt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(la[ks], __builtin_bit_cast(pf_bf16x8, hi[rt][ks]), s[rt], 0, 0, 0);
              }
          }
        }
        // the next rows (here, since the wait for Qt would be one for them too; behind the last they come once more)
        q_at = q_at == Q_AT ? Q_AT + Q_BYTES : Q_AT;
        const bool same = rg + 1 < rgs, last_head = h + 1 >= h_end;
        request_q(same || last_head ? h : h + 1, same ? rg + 1 : (last_head ? rg : 0), q_at);
        if (live) {
#pragma unroll
          for (int rt = 0; rt < 2; ++rt) {
            const int pos = first_pos + step * (min(r0 + 32 * rt + l32, n_rows - 1) / G);  // (used at the edges only)
            if (jw + 31 > pos_first) {  // some row does not see the last key
              const int last = pos - jw - 4 * g2;
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + (i & 3) > last) s[rt][i] = -INFINITY;
            }
            if (p.window > 0 && jw + p.window <= pos_last && jw + 32 > p.sinks) {  // some row's window starts behind the first key
              const int from = p.sinks - jw - 4 * g2;  // hidden: `hidden` keys from here on
              const uint32_t hidden = static_cast<uint32_t>(max(0, pos - p.window + 1 - p.sinks));
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (static_cast<uint32_t>(8 * (i >> 2) + (i & 3) - from) < hidden) s[rt][i] = -INFINITY;
            }
            const float minus = r0 + 32 * rt + l32 < n_rows ? -nl[rt] : -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] += __builtin_amdgcn_exp2f(fmaf(s[rt][i], sc, minus));
          }
        }
      }
    }
  }
  // over the 32 lanes of a half (its rows); the Q buffers serve the way to one key per lane (once the last
  // request has arrived there)
  pf_wait_vm0();
  lds_fence();
  __syncthreads();
  float* sum_s = reinterpret_cast<float*>(smem + Q_AT) + wave * 32;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v = acc[i];
    v += lane_ror<8>(v);
    v += lane_ror<4>(v);
    v += lane_ror<2>(v);
    v += lane_ror<1>(v);
    float o = v;
    permlane16_swap(v, o);
    v += o;
    if (l32 == 0) sum_s[8 * (i >> 2) + 4 * g2 + (i & 3)] = v;
  }
  __builtin_amdgcn_s_waitcnt(0xc07f);
  lds_fence();
  const int j = j0 + 32 * wave + l32;
  if (g2 == 0 && j < n_t) {
    if (gridDim.z > 1) {
      p.group_sums[(static_cast<int64_t>(blockIdx.z) * p.n_seqs + t) * p.max_seq_len + j] = sum_s[l32];
    } else {
      float* w = p.weights + t * p.weights_stride + j;
      *w = p.decay == 0.f ? sum_s[l32] : fmaf(p.decay, *w, sum_s[l32]);
    }
  }
}

// the sums of groups of heads, in the groups' order
__global__ __launch_bounds__(256) void weights_join_kernel(WeightsParams p) {
  const int t = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= min(PF_CONST_I32(p.seq_lens)[t], p.max_seq_len)) return;
  float* w = p.weights + t * p.weights_stride + j;
  float all = 0.f;
  for (int g = 0; g < p.sum_groups; ++g) all += p.group_sums[(static_cast<int64_t>(g) * p.n_seqs + t) * p.max_seq_len + j];
  *w = p.decay == 0.f ? all : fmaf(p.decay, *w, all);
}

// Few rows (32 at most per sequence and kv head: a decode step of some agents).  Waves divide the heads: a wave holds the rows
// of one in registers and walks tile_keys / 32 tiles of 32 keys, requested one ahead into LDS of its own, with no barrier before the
// workgroup's sums meet; it joins the shares' statistics of its rows itself.  (With the tiles of the kernel above three of four
// waves had no rows: 16 sequences of 4 k to 64 k tokens 282 us.)
constexpr int kSumTiles = 8;  // tiles of a wave at most
template <int D, int RP, bool HAS_BK, bool PAGED>
__global__ __launch_bounds__(256, 2) void weights_sum_rows_kernel(WeightsParams p) {
  constexpr int KS = D / 16, RKS = RP / 16, KCH = D / 8, KROWS = 64 / KCH;
  constexpr int STAGE = 32 * D * 2;
  __shared__ __align__(16) unsigned char smem[4][2 * STAGE];
  __shared__ __align__(16) float sum_s[4][kSumTiles * 32];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.y, G = p.group;
  const int j0 = blockIdx.x * p.sum_tiles * 32;
  const int n_t = min(PF_CONST_I32(p.seq_lens)[t], p.max_seq_len);
  if (j0 >= n_t) return;
  const int nt = min(p.sum_tiles, (n_t - j0 + 31) / 32);
  const int c0 = t > 0 ? min(max(PF_CONST_I32(p.seq_query_start)[t], 0), p.n_queries) : 0;
  const int c1 = t + 1 < p.n_seqs ? min(max(PF_CONST_I32(p.seq_query_start)[t + 1], c0), p.n_queries) : p.n_queries;
  const int n_rows = min((c1 - c0) * G, 32);
  const int first_pos = p.causal ? n_t - (c1 - c0) : n_t - 1;
  const int lo = p.window > 0 ? max(0, first_pos - p.window + 1) : 0, sinks = min(p.sinks, lo);
  const float sc = p.scale * 1.44269504088896340736f;
  for (int i = lane; i < nt * 32; i += 64) sum_s[wave][i] = 0.f;
  if (n_rows > 0 && wave < p.n_kv_heads && (j0 < sinks || j0 + nt * 32 > lo)) {
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem[wave])));
    const uint32_t ts2 = static_cast<uint32_t>(p.kv_token_stride) * 2u;
    uint32_t ids[2] = {0u, 0u}, id_last = 0u;
    if constexpr (PAGED) id_last = static_cast<uint32_t>(PF_CONST_I32(p.block_table)[static_cast<int64_t>(t) * p.max_blocks_per_seq + ((n_t - 1) >> 4)]);
    // the low-rank row of this lane's key, to registers (the last token's for one that nobody sees, or past the end)
    uint2 l_next[RKS][2] = {};
    auto look_up = [&](int j) __attribute__((always_inline)) {
      if constexpr (PAGED) {
        const pf_const_i32 table = PF_CONST_I32(p.block_table) + static_cast<int64_t>(t) * p.max_blocks_per_seq;
        ids[0] = static_cast<uint32_t>(table[min(j >> 4, (n_t - 1) >> 4)]);
        ids[1] = static_cast<uint32_t>(table[min((j >> 4) + 1, (n_t - 1) >> 4)]);
      }
    };
    auto kept = [&](int tok) __attribute__((always_inline)) -> bool { return tok < n_t && (tok < sinks || tok >= lo); };
    auto issue = [&](int j, int h, uint32_t at) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {  // sixteen rows at a time: one block
        const int tok = j + 16 * b;
        const bool any = tok < n_t && (tok < sinks || min(tok + 16, n_t) > lo);
        const int nv = any ? min(16, n_t - tok) : 0;
        const uint32_t bytes = nv > 0 ? static_cast<uint32_t>(nv - 1) * ts2 + D * 2 : 0u;
        const int64_t off = static_cast<int64_t>(h) * p.kv_head_stride +
                            (PAGED ? static_cast<int64_t>(ids[b]) * p.kv_block_stride : static_cast<int64_t>(tok) * p.kv_token_stride);
        const pf_u32x4 rs = pf_rsrc(static_cast<const bf16_t*>(p.k_base) + off, bytes);
#pragma unroll
        for (int i = 0; i < 16 / KROWS; ++i) {
          const int r = i * KROWS + lane / KCH;
          const uint32_t voff = static_cast<uint32_t>(r) * ts2 + ((lane % KCH ^ pf_swz_k<D>(16 * b + r)) << 4);
          pf_load16_to_lds(rs, lds0 + at + (b * (16 / KROWS) + i) * 1024, kept(tok + r) ? voff : kPfOob, 0);
        }
      }
      if constexpr (HAS_BK) {
        const int tok = kept(j + l32) ? j + l32 : n_t - 1;
        const int64_t index = PAGED ? static_cast<int64_t>(tok == j + l32 ? (l32 < 16 ? ids[0] : ids[1]) : id_last) * 16 + (tok & 15) : tok;
        const bf16_t* lr = static_cast<const bf16_t*>(p.l) + index * p.l_row_stride;
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks)
#pragma unroll
          for (int pc = 0; pc < 2; ++pc)  // (past the rank its last four again, against zeros of Qt)
            l_next[ks][pc] = *reinterpret_cast<const uint2*>(lr + min(16 * ks + 8 * pc + 4 * g2, p.rank - 4));
      }
    };
    int tok, g;
    split_row(min(l32, n_rows - 1), G, tok, g);
    const int pos = first_pos + (p.causal ? tok : 0);
    const int pos_first = __builtin_amdgcn_readfirstlane(pos), pos_last = __builtin_amdgcn_readlane(pos, 31);
    look_up(j0);
    issue(j0, wave, 0);
    uint32_t at = 0;
    for (int h = wave; h < p.n_kv_heads; h += 4) {
      // this head's rows: Q, Qt, and the reciprocal of the row sum as a logarithm
      pf_bf16x8 q[KS], hi[RKS], low[RKS];
      const int64_t row = static_cast<int64_t>(c0) * G + min(l32, n_rows - 1);
      const bf16_t* qr = static_cast<const bf16_t*>(p.q) + (static_cast<int64_t>(c0 + tok) * p.n_q_heads + h * G + g) * D + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qr + ks * 16));
      const bf16_t* qt = reinterpret_cast<const bf16_t*>(p.qt) + (static_cast<int64_t>(h) * p.rows_per_head + row) * 2 * RP + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < RKS; ++ks) {
        hi[ks] = low[ks] = pf_as_bf16x8(make_uint4(0u, 0u, 0u, 0u));
        if constexpr (HAS_BK) {
          hi[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qt + ks * 16));
          low[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qt + RP + ks * 16));
        }
      }
      float nl;
      {
        const float2* st = reinterpret_cast<const float2*>(p.stats) + static_cast<int64_t>(h) * p.n_splits * p.rows_per_head + row;
        float2 x[16];  // (at most 32 shares)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = st[static_cast<int64_t>(min(2 * i + g2, p.n_splits - 1)) * p.rows_per_head];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (2 * i + g2 < p.n_splits) m = fmaxf(m, x[i].x);
        m = fmaxf(m, pf_partner32(m));
        const float nm = m == -INFINITY ? 0.f : -m;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (2 * i + g2 < p.n_splits) l = fmaf(x[i].y, __builtin_amdgcn_exp2f(x[i].x + nm), l);
        l += pf_partner32(l);
        nl = l == 0.f || l32 >= n_rows ? -INFINITY : -(m + log2f(l));
      }
      for (int tile = 0; tile < nt; ++tile) {
        const int j = j0 + 32 * tile;
        pf_wait_vm0();
        lds_fence();
        const uint32_t now = at;
        at ^= STAGE;
        pf_bf16x8 l_op[RKS];
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks) l_op[ks] = pf_as_bf16x8(make_uint4(l_next[ks][0].x, l_next[ks][0].y, l_next[ks][1].x, l_next[ks][1].y));
        const bool wrap = tile + 1 == nt;
        const int j_next = wrap ? j0 : j + 32, h_next = wrap ? h + 4 : h;
        if (h_next < p.n_kv_heads) {
          look_up(j_next);
          issue(j_next, h_next, at);
        }
        if (!(j <= pos_last && (p.window == 0 || j + 31 + p.window > pos_first || j < p.sinks))) continue;
        const unsigned char* ks_l = smem[wave] + now;
        pf_f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        if constexpr (HAS_BK) {
#pragma unroll
          for (int ks = 0; ks < RKS; ++ks) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l_op[ks], low[ks], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(l_op[ks], hi[ks], s, 0, 0, 0);
          }
        }
        const int k_pre = l32 * (D * 2) + (pf_swz_k<D>(l32) << 4);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 a = *reinterpret_cast<const uint4*>(ks_l + (k_pre ^ ((2 * ks + g2) << 4)));
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(a), q[ks], s, 0, 0, 0);
        }
        if (j + 31 > pos_first) {
          const int last = pos - j - 4 * g2;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (8 * (i >> 2) + (i & 3) > last) s[i] = -INFINITY;
        }
        if (p.window > 0 && j + p.window <= pos_last && j + 32 > p.sinks) {
          const int from = p.sinks - j - 4 * g2;
          const uint32_t hidden = static_cast<uint32_t>(max(0, pos - p.window + 1 - p.sinks));
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (static_cast<uint32_t>(8 * (i >> 2) + (i & 3) - from) < hidden) s[i] = -INFINITY;
        }
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          v[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sc, nl));
          v[i] += lane_ror<8>(v[i]);
          v[i] += lane_ror<4>(v[i]);
          v[i] += lane_ror<2>(v[i]);
          v[i] += lane_ror<1>(v[i]);
          float o = v[i];
          permlane16_swap(v[i], o);
          v[i] += o;
        }
        if (l32 == 0) {
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            pf_f32x4* to = reinterpret_cast<pf_f32x4*>(&sum_s[wave][tile * 32 + 8 * q4 + 4 * g2]);
            *to += pf_f32x4{v[4 * q4], v[4 * q4 + 1], v[4 * q4 + 2], v[4 * q4 + 3]};
          }
        }
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < min(nt * 32, n_t - j0); i += 256) {
    float* w = p.weights + t * p.weights_stride + j0 + i;
    const float all = (sum_s[0][i] + sum_s[1][i]) + (sum_s[2][i] + sum_s[3][i]);
    *w = p.decay == 0.f ? all : fmaf(p.decay, *w, all);
  }
}

template <int D, int RP, bool HAS_BK, bool PAGED>
static void launch_passes(const WeightsParams& p, hipStream_t s) {
  hipLaunchKernelGGL((weights_stats_mfma_kernel<D, RP, HAS_BK, PAGED>), dim3(static_cast<unsigned>(p.tile_places * p.n_splits * p.n_kv_heads)), dim3(256), 0, s, p);
  if (static_cast<int64_t>(p.max_queries_per_seq) * p.group <= 32) {
    // tiles of a wave: as many as leave the chip four workgroups per compute unit (two at a time), the lengths taken for the bound
    WeightsParams q = p;
    const int64_t tiles = static_cast<int64_t>(p.n_seqs) * ((p.max_seq_len + 31) / 32);
    q.sum_tiles = static_cast<int32_t>(tiles < 1024 ? 1 : (tiles / 1024 < kSumTiles ? tiles / 1024 : kSumTiles));
    const dim3 grid((p.max_seq_len + 32 * q.sum_tiles - 1) / (32 * q.sum_tiles), p.n_seqs);
    hipLaunchKernelGGL((weights_sum_rows_kernel<D, RP, HAS_BK, PAGED>), grid, dim3(256), 0, s, q);
  } else {
    hipLaunchKernelGGL(weights_lse_kernel, dim3((p.rows_per_head + 63) / 64, p.n_kv_heads), dim3(256), 0, s, p);
    hipLaunchKernelGGL((weights_sum_mfma_kernel<D, RP, HAS_BK, PAGED>), dim3((p.max_seq_len + kSumKeys - 1) / kSumKeys, p.n_seqs, p.sum_groups), dim3(256), 0, s, p);
    if (p.sum_groups > 1) hipLaunchKernelGGL(weights_join_kernel, dim3((p.max_seq_len + 255) / 256, p.n_seqs), dim3(256), 0, s, p);
  }
}

template <int D, bool PAGED>
static void launch_by_rank(const WeightsParams& p, hipStream_t s) {
  if (p.b_k == nullptr) launch_passes<D, 16, false, PAGED>(p, s);
  else if (p.rank <= 16) launch_passes<D, 16, true, PAGED>(p, s);
  else if (p.rank <= 32) launch_passes<D, 32, true, PAGED>(p, s);
  else launch_passes<D, 64, true, PAGED>(p, s);
}

hipError_t launch_key_weights_mfma(const WeightsParams& p, hipStream_t s) {
  if (p.head_dim == 128) {
    if (p.block_size != 0) launch_by_rank<128, true>(p, s);
    else launch_by_rank<128, false>(p, s);
  } else {
    if (p.block_size != 0) launch_by_rank<64, true>(p, s);
    else launch_by_rank<64, false>(p, s);
  }
  return hipGetLastError();
}

}  // namespace lra
