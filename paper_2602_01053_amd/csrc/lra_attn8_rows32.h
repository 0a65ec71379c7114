// Attention over 8-bit codes for sequences with 17 to 64 query rows per kv head: attn8_rows_kernel with 32 rows to a wave
// (v_mfma_f32_32x32x16_bf16).  Waves of 16 rows each read every key once per row tile: 16 sequences of 4 k to 64 k tokens with 28 rows took
// 244 us so (e4m3; integers 258) and take 150 to 156 (160 to 165), 5.0 TB/s of the bytes needed; 64 rows over 32 k tokens take 38 us, as much by their
// states and products as by the reading.
//
// Operands straight from the cache, as there: row rho of key tile t (of two) is token 8 (rho / 16) + 4 (rho / 8 % 2) + rho % 4 of block
// 2t + rho / 4 % 2.  Lane half g of the result S^T then holds block 2t + g in order, register i its token i, and takes that block's 16
// bytes of a dimension of V as two operands.  Q and Qt wait in LDS, where all waves read the same operands: with them in registers there
// are too few for two waves per SIMD.
#pragma once

#include <algorithm>

#include "lra_attn8_rows.h"

namespace lra {

// Waves per SIMD that the registers leave (with two, rank 64 keeps 13 registers in scratch memory at d = 64, more at d = 128).
constexpr int attn8_rows32_waves(int rp) { return rp == 64 ? 1 : 2; }

// RT: row tiles of a workgroup (1 or 2).
template <int D, int RT, int RP, bool HAS_BK, int CODE>
__global__ __launch_bounds__(256, attn8_rows32_waves(RP)) void attn8_rows32_kernel(Batch8Params p) {
  constexpr int NS = 4 / RT;          // waves that divide the tiles of one row tile
  constexpr int KS = D / 16;          // k-steps of S^T over the head dimension
  constexpr int KW = D / 32;          // 16-byte pieces of a K row per lane: one of every two
  constexpr int DB = D / 32;          // 32-row blocks of O^T
  constexpr int RKS = RP / 16;        // k-steps over the padded rank
  constexpr int RB = (RP + 31) / 32;  // 32-row blocks of Olr^T
  constexpr int SLOT = ((DB + RB) * 16 + 1) * 64 * 4;  // a wave's state, lane by lane
  __shared__ __align__(16) unsigned char smem[2 * SLOT];
  __shared__ __align__(16) pf_u32x4 q_s[RT][KS][64];
  __shared__ __align__(16) uint4 qt_s[HAS_BK ? RT : 1][HAS_BK ? RKS : 1][64];
  __shared__ float m_s[4][32];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rt = wave % RT, stream = wave / RT;
  const int Hq = p.n_q_heads, Hkv = p.n_kv_heads, G = p.group, r = p.rank;
  int t, split, shares, h;
  if (!attn8_share(p, lane, t, split, shares, h)) return;
  const Attn8Sequence seq = attn8_sequence(p, t);
  const int n_t = seq.n_t, c0 = seq.c0, c1 = seq.c1, first_pos = seq.first_pos, lo = seq.lo, sinks = seq.sinks;
  const int sink_tiles = seq.sink_tiles, gap = seq.gap, n_tiles = seq.n_tiles, pos_last = n_t - 1;
  const int n_rows = min((c1 - c0) * G, 32 * RT);
  if (n_rows == 0) return;
  if (split == 0 && shares < p.n_splits) attn8_missing_shares(p, seq, n_rows, h, shares);
  // this lane's row (the last one again past the end)
  const int at_row = min(32 * rt + l32, n_rows - 1), tok = at_row / G;
  const int row = (c0 + tok) * Hq + h * G + (at_row - tok * G), pos = first_pos + (p.causal ? tok : 0);
  const bool live = 32 * rt + l32 < n_rows;
  const bool has_rows = 32 * rt < n_rows;  // (uniform)
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / shares);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / shares);
  const int a_first = min(max(p.query_adapter[c0], 0), p.n_adapters - 1);
  auto adapter_of_row = [&]() __attribute__((always_inline)) -> int { return p.causal ? a_first : p.query_adapter[c0 + tok]; };
  // (formed where it is used: held over the loop, it went to scratch memory)
  auto slot_of_row = [&]() __attribute__((always_inline)) -> int64_t {
    int at = row;
    asm volatile("" : "+v"(at));
    return static_cast<int64_t>(at) * p.n_splits + split;
  };
  if (t0 >= t1) {
    const int64_t slot = slot_of_row();
    // an empty state, all the merge kernel looks at; for a row that sees nothing at all share 0 leaves one that gives zeros
    if (stream == 0 && live) {
      const bool nothing = split == 0 && pos < 0;
      if (g2 == 0) {
        p.part_ml[slot * 2 + 0] = nothing ? 0.f : -INFINITY;
        p.part_ml[slot * 2 + 1] = nothing ? 1.f : 0.f;
        if (split == 0) p.part_adapter[row] = adapter_of_row();
      }
      if (nothing) {
        for (int c = g2; c < D; c += 2) p.part_o[slot * D + c] = 0.f;
        for (int c = g2; c < r; c += 2) p.part_lr[slot * r + c] = 0.f;
      }
    }
    return;
  }
  auto key_of = [&](int tile) __attribute__((always_inline)) -> int { return (tile < sink_tiles ? tile : tile + gap) * 64; };
  auto kept = [&](int key) __attribute__((always_inline)) -> bool { return key < n_t && (key < sinks || key >= lo); };
  auto whole = [&](int j) __attribute__((always_inline)) -> bool { return j + 64 <= n_t && (j + 64 <= sinks || j >= lo); };

  // ---------------- a tile's requests ----------------
  const int my_odd = (l32 >> 2) & 1;                                         // of the A operands of S^T: the tile's second block
  const int my_token = 8 * (l32 >> 4) + 4 * ((l32 >> 3) & 1) + (l32 & 3);
  const uint8_t* const kh = static_cast<const uint8_t*>(p.k_base) + h * p.kv_head_stride + my_token * D + g2 * 16;
  const uint8_t* const vh = static_cast<const uint8_t*>(p.v_base) + h * p.kv_head_stride + l32 * 16;
  const bf16_t* const lh = static_cast<const bf16_t*>(p.l) + my_token * p.l_row_stride + 8 * g2;
  // lane l: id of block l % 4 of the tile; a block that nobody sees may have any: the one of the last token stands in, weighted zero
  auto look_up = [&](int j) __attribute__((always_inline)) -> int {
    const int j0 = j + 16 * (lane & 3);
    const bool any = j0 < n_t && (j0 < sinks || j0 + 15 >= lo);
    return block8(p.block_table, p.max_blocks_per_seq, t, (any ? j0 : n_t - 1) >> 4);
  };
  auto block = [&](int id, int i) __attribute__((always_inline)) -> int64_t { return __builtin_amdgcn_readlane(id, i); };
  uint4 kc[2][KW], vc[2][DB], lc[2][RKS];
  int ks_raw, vs_raw;  // lane l: of block l % 4
  auto issue_k = [&](int id) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint8_t* src = kh + (my_odd ? block(id, 2 * kt + 1) : block(id, 2 * kt)) * p.kv_block_stride;
#pragma unroll
      for (int w = 0; w < KW; ++w) kc[kt][w] = *reinterpret_cast<const uint4*>(src + w * 32);
    }
    ks_raw = p.k_scale[id * p.scale_block_stride + h];
  };
  auto issue_l = [&](int id) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const bf16_t* src = lh + (my_odd ? block(id, 2 * kt + 1) : block(id, 2 * kt)) * 16 * p.l_row_stride;
#pragma unroll
      for (int i = 0; i < RKS; ++i) lc[kt][i] = 16 * i + 8 * g2 < r ? *reinterpret_cast<const uint4*>(src + 16 * i) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  auto issue_v = [&](int id) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint8_t* src = vh + (g2 ? block(id, 2 * kt + 1) : block(id, 2 * kt)) * p.kv_block_stride;
#pragma unroll
      for (int b = 0; b < DB; ++b) vc[kt][b] = load_once(src + b * 512);
    }
    vs_raw = p.v_scale[id * p.scale_block_stride + h];
  };
  const int first = has_rows ? t0 + stream : t1;
  int id_next = 0;
  if (first < t1) {
    const int id = look_up(key_of(first));
    issue_k(id);
    issue_l(id);
    issue_v(id);
    id_next = look_up(key_of(min(first + NS, t1 - 1)));
  }

  // ---------------- prologue: Q operands, Qt = Q B_K^T ----------------
  // lane (row l32, half g2) of k-step ks: dimensions 32 (ks / 2) + 16 g2 + 8 (ks % 2) + 0..7, the order of a lane's codes of K
  {
    const bf16_t* qr = static_cast<const bf16_t*>(p.q) + static_cast<int64_t>(row) * D + g2 * 16;
#pragma unroll
    for (int i = 0; i < KS / NS; ++i) q_s[rt][stream + NS * i][lane] = *reinterpret_cast<const pf_u32x4*>(qr + ((stream + NS * i) >> 1) * 32 + ((stream + NS * i) & 1) * 8);
  }
  __syncthreads();
  auto q_of = [&](int ks) __attribute__((always_inline)) -> bf16x8 { return __builtin_bit_cast(bf16x8, q_s[rt][ks][lane]); };
  // Qt^T, ranks by rows: register i of block b is rank 32b + 8 (i / 4) + 4 g2 + i % 4; the halves exchange fours, so that a lane has
  // ranks 16 rs + 8 g2 + 0..7 of k-step rs, as it loads them of L (in bf16, as in attn8_rows_kernel).  The waves of a row tile divide its queries (each with its adapter, or
  // the chunk's one) and hand the operands round in LDS.
  if constexpr (HAS_BK) {
    const int64_t ldb = static_cast<int64_t>(Hkv) * D;
    const int it0 = p.causal ? 0 : 32 * rt / G, it1 = !has_rows ? it0 : (p.causal ? 1 : (min(32 * rt + 32, n_rows) - 1) / G + 1);
#pragma unroll 1
    for (int it = it0 + stream; it < it1; it += NS) {
      const int a = p.causal ? a_first : min(max(p.query_adapter[c0 + it], 0), p.n_adapters - 1);
      const bf16_t* src = static_cast<const bf16_t*>(p.b_k) + static_cast<int64_t>(a) * r * ldb + h * D + g2 * 16;
#pragma unroll 1
      for (int b = 0; b < RB; ++b) {
        pf_f32x16 acc;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 bk = 32 * b + l32 < r ? *reinterpret_cast<const uint4*>(src + (32 * b + l32) * ldb + (ks >> 1) * 32 + (ks & 1) * 8) : make_uint4(0u, 0u, 0u, 0u);
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(bk), q_of(ks), acc, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (RKS == 1 && i == 1) break;
          const int o = 8 * i;
          uint32_t x[2], y[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float u = __uint_as_float(pack_bf16x2(acc[o + 2 * e], acc[o + 2 * e + 1])), w = __uint_as_float(pack_bf16x2(acc[o + 4 + 2 * e], acc[o + 5 + 2 * e]));
            permlane32_swap(u, w);
            x[e] = __float_as_uint(u), y[e] = __float_as_uint(w);
          }
          if (p.causal || tok == it) qt_s[rt][2 * b + i][lane] = make_uint4(x[0], x[1], y[0], y[1]);
        }
      }
    }
    __syncthreads();
  }
  // the identity's half i as B operand: lane (column l32), element e <-> row 8 g2 + e of the sixteen
  auto eye = [&](int i) __attribute__((always_inline)) -> bf16x8 {
    int at = l32 - 16 * i - 8 * g2;  // the element that is one
    asm volatile("" : "+v"(at));
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = at == 2 * e ? 0x3f80u : (at == 2 * e + 1 ? 0x3f800000u : 0u);
    return as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
  };

  // ---------------- main loop ----------------
  pf_f32x16 o_acc[DB], lr_acc[RB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o_acc[b][i] = 0.f;
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) lr_acc[b][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  int unit = 0;  // integers: what o_acc is counted in, a scale byte
  const float sc = p.scale * 1.44269504088896340736f;
  for (int tile = first; tile < t1; tile += NS) {
    const int j = key_of(tile);
    const bool more = tile + NS < t1;
    const bool all = whole(j);
    // S^T: register i of tile kt is token i of block 2 kt + g2
    // (from here to the next tile's requests the wave goes ahead of the SIMD's other one: 28 rows over 16 sequences 156 us instead of 159, integers 166
    // instead of 172)
    __builtin_amdgcn_s_setprio(1);
    pf_f32x16 s[2];
    {
      float ks_row[2], ks_mine[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const float even = scale8(__builtin_amdgcn_readlane(ks_raw, 2 * kt)), odd = scale8(__builtin_amdgcn_readlane(ks_raw, 2 * kt + 1));
        ks_row[kt] = my_odd ? odd : even;
        ks_mine[kt] = g2 ? odd : even;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
      }
      int at = lane;
      asm volatile("" : "+v"(at));  // (operands of Q read again for each tile, not held in registers)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 q = __builtin_bit_cast(bf16x8, q_s[rt][ks][at]);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const uint4 c = kc[kt][ks >> 1];
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(codes_to_bf16<CODE>(ks & 1 ? c.z : c.x, ks & 1 ? c.w : c.y, ks_row[kt]), q, s[kt], 0, 0, 0);
        }
      }
      if constexpr (CODE == LRA_INT8) s[0] *= ks_mine[0], s[1] *= ks_mine[1];
    }
    __builtin_amdgcn_sched_barrier(0);
    const int id_now = id_next;
    if (more) {
      issue_k(id_now);
      id_next = look_up(key_of(min(tile + 2 * NS, t1 - 1)));
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    // L: rows that nobody sees are zeros
    if (!all) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const bool in = kept(j + 32 * kt + 16 * my_odd + my_token);
#pragma unroll
        for (int i = 0; i < RKS; ++i) lc[kt][i] = in ? lc[kt][i] : make_uint4(0u, 0u, 0u, 0u);
      }
    }
    if constexpr (HAS_BK) {
      int at = lane;
      asm volatile("" : "+v"(at));
#pragma unroll
      for (int i = 0; i < RKS; ++i) {
        const bf16x8 qt = as_bf16x8(qt_s[rt][i][at]);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(lc[kt][i]), qt, s[kt], 0, 0, 0);
      }
    }
    if (j + 63 > first_pos) {  // some row does not see the last key
      const int last = pos - j - 16 * g2;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * kt + i > last) s[kt][i] = -INFINITY;
    }
    if (p.window > 0 && j + p.window <= pos_last && j + 64 > p.sinks) {  // some row's window starts behind the first key
      const int from = p.sinks - j - 16 * g2;
      const uint32_t hidden = static_cast<uint32_t>(max(0, pos - p.window + 1 - p.sinks));
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (static_cast<uint32_t>(32 * kt + i - from) < hidden) s[kt][i] = -INFINITY;
    }
    // (the accumulators are rescaled only where some row's maximum grows; the probabilities, at most 1, round to bf16 for the
    // matrix cores, their sum is taken in fp32 before)
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
    mx = tile_reference(fmaxf(mx, pf_partner32(mx)) * sc);
    if (__builtin_amdgcn_ballot_w64(mx > m_run || (CODE == LRA_INT8 && vs_raw > unit)) != 0) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
      float alpha_o = alpha;
      if constexpr (CODE == LRA_INT8) {
        int most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, __builtin_amdgcn_readlane(vs_raw, i));
        const int next = most > unit ? unit_above(most) : unit;
        alpha_o *= over_unit(unit, next);
        unit = next;
      }
#pragma unroll
      for (int b = 0; b < DB; ++b) o_acc[b] *= alpha_o;
#pragma unroll
      for (int b = 0; b < RB; ++b) lr_acc[b] *= alpha;
    }
    const float nm = m_run == -INFINITY ? 0.f : -m_run;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int vs_even = __builtin_amdgcn_readlane(vs_raw, 2 * kt), vs_odd = __builtin_amdgcn_readlane(vs_raw, 2 * kt + 1);
      // (the scale, that of e4m3 codes goes with them, or what the weights take of it)
      const float even = CODE == LRA_INT8 ? over_unit(vs_even, unit) : scale8(vs_even), odd = CODE == LRA_INT8 ? over_unit(vs_odd, unit) : scale8(vs_odd);
      const float vs_mine = g2 ? odd : even;
      uint32_t wl[8], wv[8];  // weights for L, and for V: with the block's scale, where that is not in V's operand
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[kt][2 * i], sc, nm)), y = __builtin_amdgcn_exp2f(fmaf(s[kt][2 * i + 1], sc, nm));
        l_run += x;
        l_run += y;
        wl[i] = pack_bf16x2(x, y);
        wv[i] = CODE == LRA_INT8 ? pack_bf16x2(x * vs_mine, y * vs_mine) : wl[i];  // (a power of two: the same rounding as without it)
      }
      auto half = [](const uint32_t (&w)[8], int hf) __attribute__((always_inline)) { return as_bf16x8(make_uint4(w[4 * hf], w[4 * hf + 1], w[4 * hf + 2], w[4 * hf + 3])); };
      if (!all) {  // codes of tokens that nobody sees may be no numbers: zeros
        const uint4 mask = token_masks(j + 32 * kt + 16 * g2, n_t, sinks, lo);
#pragma unroll
        for (int b = 0; b < DB; ++b) vc[kt][b] = masked(vc[kt][b], mask);
      }
      // O^T += V^T P^T: half of the sixteen tokens of both blocks
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        o_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(codes_to_bf16<CODE>(vc[kt][b].x, vc[kt][b].y, vs_mine), half(wv, 0), o_acc[b], 0, 0, 0);
        o_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(codes_to_bf16<CODE>(vc[kt][b].z, vc[kt][b].w, vs_mine), half(wv, 1), o_acc[b], 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        pf_f32x16 lt;
#pragma unroll
        for (int i = 0; i < 16; ++i) lt[i] = 0.f;
        lt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(lc[kt][2 * b]), eye(0), lt, 0, 0, 0);
        if constexpr (RKS > 1) lt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(lc[kt][RKS > 1 ? 2 * b + 1 : 0]), eye(1), lt, 0, 0, 0);
        // (bf16 values in fp32: their upper halves)
        auto pair = [&](int i) __attribute__((always_inline)) { return __builtin_amdgcn_perm(__float_as_uint(lt[i + 1]), __float_as_uint(lt[i]), 0x07060302u); };
        lr_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(pair(0), pair(2), pair(4), pair(6))), half(wl, 0), lr_acc[b], 0, 0, 0);
        lr_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(pair(8), pair(10), pair(12), pair(14))), half(wl, 1), lr_acc[b], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) {
      issue_l(id_now);
      issue_v(id_now);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // ---------------- the states of a row tile's waves: two by two through LDS, the first of them stores ----------------
  l_run += pf_partner32(l_run);
  float m_all = m_run;
  if (g2 == 0) m_s[wave][l32] = m_run;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NS; ++i) m_all = fmaxf(m_all, m_s[i * RT + rt][l32]);
  const float wgt = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_all);
  l_run = m_run == -INFINITY ? l_run : l_run * wgt;  // (a sum of NaN stays one)
#pragma unroll
  for (int b = 0; b < DB; ++b) {
    o_acc[b] *= wgt;
    if constexpr (CODE == LRA_INT8) o_acc[b] *= scale8(unit);
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) lr_acc[b] *= wgt;
#pragma unroll
  for (int stride = NS / 2; stride >= 1; stride >>= 1) {
    if (stream >= stride && stream < 2 * stride) {
      float* dst = reinterpret_cast<float*>(smem + (wave - stride * RT) * SLOT) + lane;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dst[(b * 16 + i) * 64] = o_acc[b][i];
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) dst[((DB + b) * 16 + i) * 64] = lr_acc[b][i];
      dst[(DB + RB) * 16 * 64] = l_run;
    }
    __syncthreads();
    if (stream < stride) {
      const float* src = reinterpret_cast<const float*>(smem + wave * SLOT) + lane;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o_acc[b][i] += src[(b * 16 + i) * 64];
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) lr_acc[b][i] += src[((DB + b) * 16 + i) * 64];
      l_run += src[(DB + RB) * 16 * 64];
    }
    __syncthreads();
  }
  if (stream != 0 || !live) return;
  const int64_t slot = slot_of_row();
  if (g2 == 0) {
    const bool nothing = split == 0 && pos < 0;  // (such a row's O and O_lr are zeros)
    p.part_ml[slot * 2 + 0] = nothing ? 0.f : m_all * 0.69314718055994530942f;  // natural-log units
    p.part_ml[slot * 2 + 1] = nothing ? 1.f : l_run;
    if (split == 0) p.part_adapter[row] = adapter_of_row();
  }
  // register i of a block: dimension (rank) 32 b + 8 (i / 4) + 4 g2 + i % 4
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<pf_f32x4*>(p.part_o + slot * D + 32 * b + 8 * q + 4 * g2) = pf_f32x4{o_acc[b][4 * q], o_acc[b][4 * q + 1], o_acc[b][4 * q + 2], o_acc[b][4 * q + 3]};
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int rho = 32 * b + 8 * q + 4 * g2;  // the rank is a multiple of 8: all four or none
      if (rho < r) *reinterpret_cast<pf_f32x4*>(p.part_lr + slot * r + rho) = pf_f32x4{lr_acc[b][4 * q], lr_acc[b][4 * q + 1], lr_acc[b][4 * q + 2], lr_acc[b][4 * q + 3]};
    }
}

// row_tiles: of sixteen rows, 1 (attn8_rows_kernel), 2 or 4
template <int D, int CODE>
static hipError_t launch_attn8_rows(const Batch8Params& p, int row_tiles, hipStream_t s) {
  // (with head_shares: as many as all sequences' rounding up can make of them, by eights)
  const int most = std::max(p.head_shares, (p.head_shares + 1) / 2 + p.n_seqs);
  const dim3 grid = p.head_shares > 0 ? dim3(p.n_kv_heads * ((most + 7) / 8 * 8)) : dim3(p.n_kv_heads * p.n_splits, p.n_seqs);
  auto launch = [&](auto rp_c, auto bk_c) {
    constexpr int RP = decltype(rp_c)::value;
    constexpr bool BK = decltype(bk_c)::value;
    if (row_tiles <= 1) hipLaunchKernelGGL((attn8_rows_kernel<D, RP, BK, CODE>), grid, dim3(256), 0, s, p);
    else if (row_tiles <= 2) hipLaunchKernelGGL((attn8_rows32_kernel<D, 1, RP, BK, CODE>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attn8_rows32_kernel<D, 2, RP, BK, CODE>), grid, dim3(256), 0, s, p);
  };
  auto by_rank = [&](auto bk_c) {
    if (p.rank <= 16) launch(std::integral_constant<int, 16>{}, bk_c);
    else if (p.rank <= 32) launch(std::integral_constant<int, 32>{}, bk_c);
    else launch(std::integral_constant<int, 64>{}, bk_c);
  };
  if (p.b_k != nullptr) by_rank(std::true_type{});
  else by_rank(std::false_type{});
  return hipGetLastError();
}

}  // namespace lra
