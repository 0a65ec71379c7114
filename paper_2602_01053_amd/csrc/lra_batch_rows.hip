// Attention of a batch whose sequences have few query rows (bf16, gfx950): 32 at most per kv head, a decode step of some agents or a
// few tokens, through a window and sinks or not.
//
// One workgroup streams a share of one (sequence, kv head)'s visible keys for all its rows; its four waves take 32-key tiles in turn
// and are on their own from the first tile to the last, each with room for one in LDS:
//   S^T = K_base Q^T + L Qt^T,  online softmax along keys,  O^T += V_base^T P^T,  Olr^T += L^T P^T       (v_mfma_f32_32x32x16_bf16)
// K of the next tile is requested as soon as the scores are taken, V and L as soon as the products are, so that a compute unit's eight
// waves keep some hundred KB on their way (the tile-walking kernel's workgroups wait for the slowest of 36 requests at every tile, and
// three of their four waves have no rows: 16 sequences of 4 agents behind a window of 8 k, 87 us there).  The waves' states meet in
// LDS at the end, one state per row and share goes to the workspace.
#include "lra_batch.h"
#include "lra_decode_util.h"
#include "lra_prefill_util.h"

namespace lra {

constexpr int kRowsLds = 80 * 1024;  // half of a compute unit's LDS

template <int D, int RP, bool HAS_BK, bool PAGED>
__global__ __launch_bounds__(256, 2) void batch_rows_kernel(BatchParams p) {
  constexpr int KS = D / 16, RKS = RP / 16, DB = D / 32, RB = (RP + 31) / 32;
  constexpr int KCH = D / 8, KROWS = 64 / KCH, LCH = RP / 8, LROWS = 64 / LCH;
  constexpr int K_BYTES = 32 * D * 2, L_BYTES = 32 * RP * 2, WAVE = 2 * K_BYTES + L_BYTES;
  constexpr int NK = 32 / KROWS, NV = NK, NL = LCH / 2;  // requests of a tile
  constexpr int SLOT = ((DB + RB) * 16 + 1) * 64 * 4;    // a wave's state, lane by lane
  constexpr int SMEM = 4 * WAVE > 2 * SLOT ? 4 * WAVE : 2 * SLOT;
  // Two workgroups to a compute unit, as the plan counts them: where the tiles alone take half of its LDS (d = 128, ranks above 32), Qt
  // passes through the last wave's V tile before that is requested, and the maxima through the K tiles behind the loop.  (One workgroup to
  // a unit, rank 64: 4 agents on 32 k tokens 48 us against 38, behind a window of 4 k 25 against 18, 16 sequences behind 8 k 78 against 70.)
  constexpr bool TIGHT = SMEM + 4 * 32 * 4 + (HAS_BK ? RKS * 1024 : 0) > kRowsLds;
  constexpr int QT_AT = 3 * WAVE + K_BYTES;
  static_assert(!TIGHT || (SMEM <= kRowsLds && RKS * 1024 <= K_BYTES && 4 * WAVE == SMEM));
  __shared__ __align__(16) unsigned char smem[SMEM];
  __shared__ float m_own[TIGHT ? 1 : 4][32];
  __shared__ __align__(16) pf_u32x4 qt_own[HAS_BK && !TIGHT ? RKS : 1][64];
  auto m_s = [&](int w) __attribute__((always_inline)) -> float* { return TIGHT ? reinterpret_cast<float*>(smem + w * WAVE) : m_own[w]; };
  auto qt_s = [&](int ks) __attribute__((always_inline)) -> pf_u32x4* {
    return TIGHT ? reinterpret_cast<pf_u32x4*>(smem + QT_AT) + ks * 64 : qt_own[ks];
  };
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hq = p.n_q_heads, Hkv = p.n_kv_heads, G = p.group, r = p.rank;
  const int split = blockIdx.x / Hkv, h = blockIdx.x - split * Hkv, t = blockIdx.y;  // (kv head fastest: one XCD, where there are eight)
  const int n_t = min(PF_CONST_I32(p.seq_lens)[t], p.max_seq_len);
  const int c0 = t > 0 ? min(max(PF_CONST_I32(p.seq_query_start)[t], 0), p.n_queries) : 0;
  const int c1 = t + 1 < p.n_seqs ? min(max(PF_CONST_I32(p.seq_query_start)[t + 1], c0), p.n_queries) : p.n_queries;
  const int n_rows = min((c1 - c0) * G, 32);
  if (n_rows == 0) return;
  // this lane's row (the last one again past the end)
  const int at_row = min(l32, n_rows - 1), tok = at_row / G, gq = at_row - tok * G;
  const int first_pos = p.causal ? n_t - (c1 - c0) : n_t - 1;
  const int pos = first_pos + (p.causal ? tok : 0);
  const int pos_last = n_t - 1;
  const int out_row = l32 < n_rows ? (c0 + tok) * Hq + h * G + gq : -1;
  const int64_t slot = static_cast<int64_t>((c0 + tok) * Hq + h * G + gq) * p.n_splits + split;
  const int lo = p.window > 0 ? max(0, first_pos - p.window + 1) : 0, sinks = min(p.sinks, lo);
  const int sink_tiles = (sinks + 31) / 32, gap = max(0, lo / 32 - sink_tiles);
  const int n_tiles = n_t <= 0 ? 0 : (n_t - 1) / 32 + 1 - gap;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / p.n_splits);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / p.n_splits);
  const int a_first = min(max(PF_CONST_I32(p.query_adapter)[c0], 0), p.n_adapters - 1);
  auto adapter_of_row = [&]() __attribute__((always_inline)) -> int { return p.causal ? a_first : p.query_adapter[c0 + tok]; };
  if (t0 >= t1) {
    // an empty state, all the merge kernel looks at; for a row that sees nothing at all share 0 leaves one that gives zeros
    if (wave == 0 && out_row >= 0) {
      const bool nothing = split == 0 && pos < 0;
      if (g2 == 0) {
        p.part_ml[slot * 2 + 0] = nothing ? 0.f : -INFINITY;
        p.part_ml[slot * 2 + 1] = nothing ? 1.f : 0.f;
        if (split == 0) p.part_adapter[out_row] = adapter_of_row();
      }
      if (nothing) {
        for (int c = g2; c < D; c += 2) p.part_o[slot * D + c] = 0.f;
        for (int c = g2; c < r; c += 2) p.part_lr[slot * r + c] = 0.f;
      }
    }
    return;
  }
  auto key_of = [&](int tile) __attribute__((always_inline)) -> int { return (tile < sink_tiles ? tile : tile + gap) * 32; };

  // ---------------- a tile's requests (rows that nobody sees lie outside the resource; their blocks may have any id) ----------------
  unsigned char* const mine = smem + wave * WAVE;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, mine)));
  const uint32_t ts2 = static_cast<uint32_t>(p.kv_token_stride) * 2u, lp2 = static_cast<uint32_t>(p.l_row_stride) * 2u;
  const uint32_t l_rows = PAGED ? static_cast<uint32_t>(p.num_blocks) * 16u : static_cast<uint32_t>(n_t);
  const pf_u32x4 rs_l = pf_rsrc(static_cast<const bf16_t*>(p.l) + static_cast<int64_t>(p.l_adapter_stride > 0 ? a_first : 0) * p.l_adapter_stride,
                                (l_rows - 1u) * lp2 + static_cast<uint32_t>(r) * 2u);
  uint32_t ids[2] = {0u, 0u};
  auto look_up = [&](int j) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      const pf_const_i32 table = PF_CONST_I32(p.block_table) + static_cast<int64_t>(t) * p.max_blocks_per_seq;
      ids[0] = static_cast<uint32_t>(table[min(j >> 4, (n_t - 1) >> 4)]);
      ids[1] = static_cast<uint32_t>(table[min((j >> 4) + 1, (n_t - 1) >> 4)]);
    }
  };
  auto kept = [&](int key) __attribute__((always_inline)) -> bool { return key < n_t && (key < sinks || key >= lo); };
  auto issue_rows = [&](const void* base, int j, uint32_t at, auto swz) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {  // sixteen rows at a time: one block
      const int key = j + 16 * b;
      const bool any = key < n_t && (key < sinks || min(key + 16, n_t) > lo);
      const int nv = any ? min(16, n_t - key) : 0;
      const uint32_t bytes = nv > 0 ? static_cast<uint32_t>(nv - 1) * ts2 + D * 2 : 0u;
      const int64_t off = static_cast<int64_t>(h) * p.kv_head_stride +
                          (PAGED ? static_cast<int64_t>(ids[b]) * p.kv_block_stride : static_cast<int64_t>(key) * p.kv_token_stride);
      const pf_u32x4 rs = pf_rsrc(static_cast<const bf16_t*>(base) + off, bytes);
#pragma unroll
      for (int i = 0; i < 16 / KROWS; ++i) {
        const int row = i * KROWS + lane / KCH;
        const uint32_t voff = static_cast<uint32_t>(row) * ts2 + ((lane % KCH ^ swz(16 * b + row)) << 4);
        pf_load16_to_lds(rs, lds0 + at + (b * (16 / KROWS) + i) * 1024, kept(key + row) ? voff : kPfOob, 0);
      }
    }
  };
  auto issue_k = [&](int j) __attribute__((always_inline)) { issue_rows(p.k_base, j, 0, [](int row) { return pf_swz_k<D>(row); }); };
  auto issue_v = [&](int j) __attribute__((always_inline)) { issue_rows(p.v_base, j, K_BYTES, [](int row) { return pf_swz_v<D>(row); }); };
  auto issue_l = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = i * LROWS + lane / LCH, key = j + row;
      const uint32_t index = PAGED ? (row < 16 ? ids[0] : ids[1]) * 16u + (static_cast<uint32_t>(key) & 15u) : static_cast<uint32_t>(key);
      const int ch = lane % LCH ^ pf_swz_l<LCH>(row);
      pf_load16_to_lds(rs_l, lds0 + 2 * K_BYTES + i * 1024, kept(key) && ch * 8 < r ? index * lp2 + (ch << 4) : kPfOob, 0);
    }
  };
  const int first = t0 + wave;
  const bool v_late = TIGHT && HAS_BK && wave == 3;
  if (first < t1) {
    look_up(key_of(first));
    issue_k(key_of(first));
    issue_l(key_of(first));
    if (!v_late) issue_v(key_of(first));
  }

  // ---------------- prologue: Q operands, Qt = Q B_K^T (as in batch_tiles_body) ----------------
  pf_bf16x8 qb[KS], qtb[RKS];
  {
    const bf16_t* qr = static_cast<const bf16_t*>(p.q) + static_cast<int64_t>((c0 + tok) * Hq + h * G + gq) * D + g2 * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qb[ks] = pf_as_bf16x8(*reinterpret_cast<const uint4*>(qr + ks * 16));
  }
  // The waves divide the adapters (of every query, or the chunk's one) and hand the operands round in LDS: with all four forming all
  // of them four agents' call on 4 k keys took 2 us longer.
  if constexpr (HAS_BK) {
    const int64_t ldb = static_cast<int64_t>(Hkv) * D;
    const bf16_t* bkg = static_cast<const bf16_t*>(p.b_k) + h * D;
    const int n_it = p.causal ? 1 : (n_rows - 1) / G + 1;
#pragma unroll 1
    for (int it = wave; it < n_it; it += 4) {
      const int a = p.causal ? a_first : min(max(PF_CONST_I32(p.query_adapter)[c0 + it], 0), p.n_adapters - 1);
      const __amdgpu_buffer_rsrc_t rs_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(bkg) + static_cast<int64_t>(a) * r * ldb, 0,
                                                                            static_cast<int>((static_cast<int64_t>(r - 1) * ldb + D) * 2), 0x00020000);
      pf_u32x4 bk[RB][KS];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int rho = b * 32 + l32;
        const uint32_t boff = rho < r ? static_cast<uint32_t>(rho * ldb * 2 + g2 * 16) : kPfOob;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) bk[b][ks] = __builtin_amdgcn_raw_buffer_load_b128(rs_b, boff, ks * 32, 0);
      }
      pf_f32x16 acc[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pf_bf16x8, bk[b][ks]), qb[ks], acc[b], 0, 0, 0);
      }
      if (p.causal || tok == it) {
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks) {
          const pf_f32x16& c = acc[ks >> 1];
          const int o = (ks & 1) * 8;
          qt_s(ks)[lane] = pf_u32x4{pf_pack2(c[o + 0], c[o + 1]), pf_pack2(c[o + 2], c[o + 3]), pf_pack2(c[o + 4], c[o + 5]), pf_pack2(c[o + 6], c[o + 7])};
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < RKS; ++ks) qtb[ks] = __builtin_bit_cast(pf_bf16x8, qt_s(ks)[lane]);
    if constexpr (TIGHT) {
      __syncthreads();  // (everyone has its operands)
      lds_fence();
      if (v_late && first < t1) issue_v(key_of(first));
    }
  }

  // ---------------- per-lane LDS read offsets (see batch_tiles_body) ----------------
  const int k_pre = l32 * (D * 2) + (pf_swz_k<D>(l32) << 4);
  const int a16 = lane & 15, dsel = (lane >> 4) & 1;
  const int vrow = 4 * g2 + (a16 >> 2);
  const int v_pre = K_BYTES + vrow * (D * 2) + ((((a16 & 3) >> 1) + 2 * dsel + pf_swz_v<D>(vrow)) << 4) + (a16 & 1) * 8;
  const int l_pre = 2 * K_BYTES + l32 * (RP * 2) + (pf_swz_l<LCH>(l32) << 4) + g2 * 8;  // (chunk c at l_pre ^ (c << 4))
  int lt_rd[RB][2];
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int key = vrow + 8 * hh, ch = 4 * b + 2 * dsel + ((a16 & 3) >> 1);
      lt_rd[b][hh] = 2 * K_BYTES + key * (RP * 2) + (((ch & (LCH - 1)) ^ pf_swz_l<LCH>(key)) << 4) + (a16 & 1) * 8;
    }

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
  const float sc = p.scale * 1.44269504088896340736f;
  for (int tile = first; tile < t1; tile += 4) {
    const int j = key_of(tile);
    const bool more = tile + 4 < t1;
    const int j_next = key_of(tile + 4);
    wait_vm<NV>();  // K and L of this tile are here, V may be on its way
    lds_fence();
    if (more) look_up(j_next);
    pf_f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4 a = *reinterpret_cast<const uint4*>(mine + (k_pre ^ ((2 * ks + g2) << 4)));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(a), qb[ks], s, 0, 0, 0);
    }
    if constexpr (HAS_BK) {
      int l_at = l_pre;
      if constexpr (TIGHT) asm volatile("" : "+v"(l_at));  // (addresses formed again for each tile: held in registers they went to scratch memory)
#pragma unroll
      for (int ks = 0; ks < RKS; ++ks) {
        const uint2 x = *reinterpret_cast<const uint2*>(mine + (l_at ^ ((2 * ks) << 4)));
        const uint2 y = *reinterpret_cast<const uint2*>(mine + (l_at ^ ((2 * ks + 1) << 4)));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(make_uint4(x.x, x.y, y.x, y.y)), qtb[ks], s, 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the K rows have been read
    lds_fence();
    if (more) issue_k(j_next);
    if (j + 31 > first_pos) {  // some row does not see the last key
      const int last = pos - j - 4 * g2;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) > last) s[i] = -INFINITY;
    }
    if (p.window > 0 && j + p.window <= pos_last && j + 32 > p.sinks) {  // some row's window starts behind the first key
      const int from = p.sinks - j - 4 * g2;
      const uint32_t hidden = static_cast<uint32_t>(max(0, pos - p.window + 1 - p.sinks));
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (static_cast<uint32_t>(8 * (i >> 2) + (i & 3) - from) < hidden) s[i] = -INFINITY;
    }
    // (the accumulators are rescaled only where some row's maximum grows; the probabilities, at most 1, round to bf16 for the
    // matrix cores, their sum is taken in fp32 before)
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = tile_reference(fmaxf(mx, pf_partner32(mx)) * sc);
    if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int b = 0; b < DB; ++b) o_acc[b] *= alpha;
#pragma unroll
      for (int b = 0; b < RB; ++b) lr_acc[b] *= alpha;
    }
    const float nm = m_run == -INFINITY ? 0.f : -m_run;
    float e[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sc, nm));
      l_run += e[i];
    }
    pf_bf16x8 pb[2];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
      pb[h2] = pf_as_bf16x8(make_uint4(pf_pack2(e[8 * h2 + 0], e[8 * h2 + 1]), pf_pack2(e[8 * h2 + 2], e[8 * h2 + 3]),
                                       pf_pack2(e[8 * h2 + 4], e[8 * h2 + 5]), pf_pack2(e[8 * h2 + 6], e[8 * h2 + 7])));
    if (more) wait_vm<NK>();  // V of this tile is here, K of the next may be on its way
    else pf_wait_vm0();
    lds_fence();
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const unsigned char* src = mine + (v_pre ^ (b << 6)) + 16 * h2 * (D * 2);
        o_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_join(pf_read_tr16(src), pf_read_tr16(src + 8 * (D * 2))), pb[h2], o_acc[b], 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b)
        lr_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            pf_join(pf_read_tr16(mine + lt_rd[b][0] + 16 * h2 * (RP * 2)), pf_read_tr16(mine + lt_rd[b][1] + 16 * h2 * (RP * 2))), pb[h2], lr_acc[b], 0, 0, 0);
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // V and L have been read
    lds_fence();
    if (more) {
      issue_l(j_next);
      issue_v(j_next);
    }
  }

  // ---------------- the waves' states: two by two through LDS, wave 0 stores ----------------
  l_run += pf_partner32(l_run);
  if (g2 == 0) m_s(wave)[l32] = m_run;
  __syncthreads();
  const float m_all = fmaxf(fmaxf(m_s(0)[l32], m_s(1)[l32]), fmaxf(m_s(2)[l32], m_s(3)[l32]));
  if constexpr (TIGHT) __syncthreads();  // (the states go where these were)
  const float wgt = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_all);
  l_run = m_run == -INFINITY ? l_run : l_run * wgt;  // (a sum of NaN stays one)
#pragma unroll
  for (int b = 0; b < DB; ++b) o_acc[b] *= wgt;
#pragma unroll
  for (int b = 0; b < RB; ++b) lr_acc[b] *= wgt;
#pragma unroll
  for (int stride = 2; stride >= 1; stride >>= 1) {
    if (wave >= stride && wave < 2 * stride) {
      float* dst = reinterpret_cast<float*>(smem + (wave - stride) * SLOT) + lane;
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
    if (wave < stride) {
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
  if (wave != 0 || out_row < 0) return;
  if (g2 == 0) {
    const bool nothing = split == 0 && pos < 0;  // (such a row's O and O_lr are zeros)
    p.part_ml[slot * 2 + 0] = nothing ? 0.f : m_all * 0.69314718055994530942f;  // natural-log units
    p.part_ml[slot * 2 + 1] = nothing ? 1.f : l_run;
    if (split == 0) p.part_adapter[out_row] = adapter_of_row();
  }
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<pf_f32x4*>(p.part_o + slot * D + 32 * b + 8 * q + 4 * g2) =
          pf_f32x4{o_acc[b][4 * q + 0], o_acc[b][4 * q + 1], o_acc[b][4 * q + 2], o_acc[b][4 * q + 3]};
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int rho = 32 * b + 8 * q + 4 * g2;  // the rank is a multiple of 8: all four or none
      if (rho < r)
        *reinterpret_cast<pf_f32x4*>(p.part_lr + slot * r + rho) =
            pf_f32x4{lr_acc[b][4 * q + 0], lr_acc[b][4 * q + 1], lr_acc[b][4 * q + 2], lr_acc[b][4 * q + 3]};
    }
}

template <int D, int RP>
static void launch_rows(const BatchParams& p, hipStream_t s) {
  const dim3 grid(p.n_kv_heads * p.n_splits, p.n_seqs);
  const bool paged = p.block_size != 0, has_bk = p.b_k != nullptr;
  if (paged && has_bk) hipLaunchKernelGGL((batch_rows_kernel<D, RP, true, true>), grid, dim3(256), 0, s, p);
  else if (paged) hipLaunchKernelGGL((batch_rows_kernel<D, RP, false, true>), grid, dim3(256), 0, s, p);
  else if (has_bk) hipLaunchKernelGGL((batch_rows_kernel<D, RP, true, false>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((batch_rows_kernel<D, RP, false, false>), grid, dim3(256), 0, s, p);
}

hipError_t launch_batch_rows(const BatchParams& p, hipStream_t s) {
  if (p.head_dim == 128) {
    if (p.rank <= 16) launch_rows<128, 16>(p, s);
    else if (p.rank <= 32) launch_rows<128, 32>(p, s);
    else launch_rows<128, 64>(p, s);
  } else {
    if (p.rank <= 16) launch_rows<64, 16>(p, s);
    else if (p.rank <= 32) launch_rows<64, 32>(p, s);
    else launch_rows<64, 64>(p, s);
  }
  return hipGetLastError();
}

}  // namespace lra
