// Tile-walking attention of a batch (bf16, gfx950): the prefill kernel's tile (lra_prefill_mfma.hip) for the chunks of many
// sequences, each with its own adapter, seen through a window and sinks.
//
// A workgroup of four waves owns 128 query rows of one sequence and kv head, a row being a new token of one of the q heads of
// the group, and walks 64-key tiles that the waves share:
//   S^T = K_base Q^T + L Qt^T,  online softmax along keys,  O^T += V_base^T P^T,  Olr^T += L^T P^T        (MFMA)
// What differs from the prefill of one sequence: the tile's sequence is found on the device (batch_tiles); tiles between the
// sinks and the window are passed over, rows of a tile that nothing in it sees read as zeros and touch no memory; a row may
// see nothing of a tile, or nothing at all.  Text of its own and not a form of that kernel: its 136 instantiations are
// scheduled to the register, and a change of their text moved 54 of them.
//
// HAS_BK: a key-side adapter by Qt = Q B_K^T; ROPE_K: one that is rotated by the key's position, added to every K tile in LDS.
// SPLIT: the key tiles of a q tile are shared by gridDim.y workgroups, whose states the merge kernel joins.
// POOL: a paged cache within 32-bit byte offsets.
#pragma once

#include "lra_batch.h"
#include "lra_prefill_util.h"

namespace lra {

// Tile traffic: HBM -> LDS with no registers in between, layout and swizzles as in PfTileLoader (lra_prefill_util.h).  Tokens
// from cut_lo to cut_hi - 1, between sinks and window, are left out: their rows lie outside the resource, and blocks that hold
// no others may have any id in the table (block 0 stands in, of which nothing is read).
template <int D, int RP, bool PAGED, bool POOL>
struct BatchTileLoader {
  static constexpr int BN = 64;
  static constexpr int KCH = D / 8;              // 16-byte chunks per K/V row
  static constexpr int KROWS = 64 / KCH;         // K/V rows one wave-wide load moves (4 or 8)
  static constexpr int KV_DMA = BN / KROWS / 4;  // wave-wide loads per wave and K (or V) tile (4 or 2)
  static constexpr int LCH = RP / 8;             // 16-byte chunks per L row (2, 4 or 8)
  static constexpr int LROWS = 64 / LCH;         // L rows one wave-wide load moves (32, 16 or 8)
  static constexpr int L_DMA = (LCH + 3) / 4;    // the tile takes LCH loads; wave w issues i = w + 4q < LCH
  static constexpr int K_BYTES = BN * D * 2;

  const Params& p;
  const bf16_t *kb, *vb;
  pf_u32x4 rs_k, rs_v, rs_l;
  uint32_t ts2, r2, lp2, lds0, k_voff, v_voff, l_voff[L_DMA];  // lp2: bytes between L rows
  int wave, lane, hk, seq, n_t, nb_last;
  int cut_lo, cut_hi;
  __device__ __forceinline__ bool kept(int tok) const { return tok < cut_lo || tok >= cut_hi; }
  __device__ __forceinline__ bool cuts(int j) const { return j < cut_hi && j + BN > cut_lo; }  // the tile at j has rows left out
  // Paged cache: the block ids of an aligned group of 64 blocks (16 tiles), lane l holding that of block l of the
  // group.  A tile takes its four by v_readlane.  (Looked up by scalar loads where the requests are formed, every
  // tile began with a memory round trip: 1.29 against 1.07 us per tile on a unit of its own, that of contiguous rows.)
  mutable int ids = 0;
  // reads the ids of the group of block b (clamped to the sequence's last block)
  __device__ __forceinline__ void fetch_ids(int b) const {
    const int at = min((b & ~63) + lane, nb_last);
    const int id = p.block_table[static_cast<int64_t>(seq) * p.max_blocks_per_seq + at];
    ids = at * 16 < cut_lo || at * 16 + 15 >= cut_hi ? id : 0;
  }
  __device__ __forceinline__ int block_id(int b) const { return __builtin_amdgcn_readlane(ids, b & 63); }

  __device__ __forceinline__ BatchTileLoader(const Params& p_, unsigned char* smem, int wave_, int lane_, int hk_, int t, int n_t_,
                                             int adapter, int cut_lo_, int cut_hi_)
      : p(p_), wave(wave_), lane(lane_), hk(hk_), seq(t), n_t(n_t_), cut_lo(cut_lo_), cut_hi(cut_hi_) {
    kb = static_cast<const bf16_t*>(p.k_base);
    vb = static_cast<const bf16_t*>(p.v_base);
    // the rows of the tile's one adapter (BaseShared: its own low-rank cache), with their own stride
    const bf16_t* lr = static_cast<const bf16_t*>(p.l) + static_cast<int64_t>(adapter) * p.l_adapter_stride;
    const int r = p.rank;
    ts2 = static_cast<uint32_t>(p.kv_token_stride) * 2u;
    r2 = static_cast<uint32_t>(r) * 2u;
    lp2 = static_cast<uint32_t>(p.l_row_stride) * 2u;
    lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem)));
    nb_last = (n_t - 1) >> 4;
    const int rr = lane / KCH, pc = lane % KCH;
    const int krow = wave * KROWS + rr;  // LDS row of load i = w (loads w + 4q: + 4q*KROWS, same swizzle)
    k_voff = static_cast<uint32_t>(rr) * ts2 + ((pc ^ pf_swz_k<D>(krow)) << 4);
    v_voff = static_cast<uint32_t>(rr) * ts2 + ((pc ^ pf_swz_v<D>(krow)) << 4);
    rs_k = rs_v = rs_l = pf_u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int q = 0; q < L_DMA; ++q) l_voff[q] = kPfOob;
    if (!PAGED) {
      const uint32_t kv_bytes = static_cast<uint32_t>(n_t - 1) * ts2 + D * 2;
      rs_k = pf_rsrc(kb + static_cast<int64_t>(hk) * p.kv_head_stride, kv_bytes);
      rs_v = pf_rsrc(vb + static_cast<int64_t>(hk) * p.kv_head_stride, kv_bytes);
      rs_l = pf_rsrc(lr, static_cast<uint32_t>(n_t - 1) * lp2 + r2);
#pragma unroll
      for (int q = 0; q < L_DMA; ++q) {
        const int lrow = (wave + 4 * q) * LROWS + lane / LCH;
        const int lch = (lane % LCH) ^ pf_swz_l<LCH>(lrow);
        l_voff[q] = (lch * 8 < r) ? static_cast<uint32_t>(lane / LCH) * lp2 + (lch << 4) : kPfOob;
      }
    } else {
      if (POOL) {
        const int64_t hoff = static_cast<int64_t>(hk) * p.kv_head_stride;
        // (every block lies below that size, kPfOob beyond it)
        rs_k = pf_rsrc(kb + hoff, kPfPoolBytes);
        rs_v = pf_rsrc(vb + hoff, kPfPoolBytes);
      }
      // paged L: one resource over the whole array; the lane's physical row is chosen per tile
      rs_l = pf_rsrc(lr, (static_cast<uint32_t>(p.num_blocks) * 16u - 1u) * lp2 + r2);
    }
  }

  // K and V loads number q (of KV_DMA) of this wave for the tile starting at key j
  __device__ __forceinline__ void issue_kv(int j, uint32_t stage_off, int q) const {
    const int i = wave + 4 * q;
    const uint32_t dst = lds0 + stage_off + i * 1024;
    if (!PAGED) {
      const uint32_t soff = static_cast<uint32_t>(j + i * KROWS) * ts2;
      if (cuts(j)) {
        const bool ok = kept(j + i * KROWS + lane / KCH);
        pf_load16_to_lds(rs_k, dst, ok ? k_voff : kPfOob, soff);
        pf_load16_to_lds(rs_v, dst + K_BYTES, ok ? v_voff : kPfOob, soff);
      } else {
        pf_load16_to_lds(rs_k, dst, k_voff, soff);
        pf_load16_to_lds(rs_v, dst + K_BYTES, v_voff, soff);
      }
    } else if (POOL) {
      // one resource per pool: a load is a multiplication and an addition away from its block id.  The rows of one
      // load lie in one 16-token block; those past the end of the sequence are cut by the lane's offset.
      const int tok = j + i * KROWS;
      const bool ok = tok + lane / KCH < n_t && kept(tok + lane / KCH);
      const uint32_t bs2 = static_cast<uint32_t>(p.kv_block_stride) * 2u;
      const uint32_t in_blk = static_cast<uint32_t>(tok & 15) * ts2;
      const uint32_t soff = static_cast<uint32_t>(block_id(tok >> 4)) * bs2 + in_blk;
      pf_load16_to_lds(rs_k, dst, ok ? k_voff : kPfOob, soff);
      pf_load16_to_lds(rs_v, dst + K_BYTES, ok ? v_voff : kPfOob, soff);
    } else {
      // the KROWS rows of one load lie in one 16-token block
      const int tok = j + i * KROWS;
      const int blk = block_id(tok >> 4);
      const int nv = max(0, min(KROWS, n_t - tok));  // rows of this load inside the sequence
      const uint32_t bytes = nv > 0 ? static_cast<uint32_t>(nv - 1) * ts2 + D * 2 : 0u;
      const int64_t off = static_cast<int64_t>(blk) * p.kv_block_stride + static_cast<int64_t>(hk) * p.kv_head_stride +
                          static_cast<int64_t>(tok & 15) * p.kv_token_stride;
      const bool ok = !cuts(j) || kept(tok + lane / KCH);
      pf_load16_to_lds(pf_rsrc(kb + off, bytes), dst, ok ? k_voff : kPfOob, 0);
      pf_load16_to_lds(pf_rsrc(vb + off, bytes), dst + K_BYTES, ok ? v_voff : kPfOob, 0);
    }
  }

  __device__ __forceinline__ void issue_l(int j, uint32_t stage_off) const {
    const int r = p.rank;
#pragma unroll
    for (int q = 0; q < L_DMA; ++q) {
      const int i = wave + 4 * q;
      if (i < LCH) {
        const uint32_t dst = lds0 + stage_off + 2 * K_BYTES + i * 1024;
        if (!PAGED) {
          const bool ok = !cuts(j) || kept(j + i * LROWS + lane / LCH);
          pf_load16_to_lds(rs_l, dst, ok ? l_voff[q] : kPfOob, static_cast<uint32_t>(j + i * LROWS) * lp2);
        } else {
          // LROWS rows span at most two blocks
          const int tok0 = j + i * LROWS;
          const int blk_a = block_id(tok0 >> 4);
          const int blk_b = LROWS > 16 ? block_id((tok0 >> 4) + 1) : blk_a;  // (16 rows or fewer lie in one block)
          const int lrow = i * LROWS + lane / LCH;
          const int tok = tok0 + lane / LCH;
          const int blk = ((tok >> 4) == (tok0 >> 4)) ? blk_a : blk_b;
          const int lch = (lane % LCH) ^ pf_swz_l<LCH>(lrow);
          const uint32_t voff = (tok < n_t && kept(tok) && lch * 8 < r)
                                    ? (static_cast<uint32_t>(blk) * 16u + static_cast<uint32_t>(tok & 15)) * lp2 + (lch << 4)
                                    : kPfOob;
          pf_load16_to_lds(rs_l, dst, voff, 0);
        }
      }
    }
  }

  // this wave's share of the tile starting at key j, into the stage at byte offset stage_off
  __device__ __forceinline__ void issue_tile(int j, uint32_t stage_off) const {
#pragma unroll
    for (int q = 0; q < KV_DMA; ++q) issue_kv(j, stage_off, q);
    issue_l(j, stage_off);
    // the ids of the next sixteen tiles travel behind the requests of the last of this sixteen
    if (PAGED && (((j >> 4) + 4) & 63) == 0) fetch_ids((j >> 4) + 4);
  }
};


template <int D, int RP, bool PAGED, bool POOL, bool HAS_BK, bool SPLIT, bool ROPE_K>
__device__ __forceinline__ void batch_tiles_body(const BatchParams p) {
  static_assert(!(ROPE_K && HAS_BK), "the rotary key side replaces the Qt term");
  // Keys completed with their rotated adapter part, K_base + RoPE(L B_K), are held as fp16: rounding the sum to bf16 a
  // second time costs 2.5e-3 to 4e-3 of relative error in the output on its own, fp16 (three more bits) a quarter of that.
  // The scores are then an fp16 product, with Q converted once in the prologue (exact for a bf16 Q of
  // ordinary magnitudes); V, L and the probabilities stay bf16.
  constexpr bool KF16 = ROPE_K;
  constexpr int BM = 128, BN = 64;
  constexpr int KS = D / 16;   // k-steps of S^T over the head dimension
  constexpr int RKS = RP / 16; // k-steps over the padded rank
  constexpr int DB = D / 32;   // 32-row blocks of O^T
  constexpr int RB = (RP + 31) / 32;  // 32-row blocks of Olr^T
  constexpr int KCH = D / 8;          // 16-byte chunks per K/V row
  constexpr int LCH = RP / 8;         // 16-byte chunks per L row (2, 4 or 8)
  constexpr int K_BYTES = BN * D * 2;
  constexpr int L_BYTES = BN * RP * 2;
  constexpr int STAGE = 2 * K_BYTES + L_BYTES;
  // With a half-empty last 32-row block of Olr^T (rank 16 or 48 after padding), its idle
  // upper lanes read a constant [1, 0, 0, 0] instead of L, so the matrix core also
  // accumulates the softmax row sums.
  constexpr bool ONES_ROW = (RP % 32) != 0;
  constexpr int ONES_AT = 2 * STAGE;

  __shared__ __align__(16) unsigned char smem[2 * STAGE + (ONES_ROW ? 16 : 0)];
  // rotary key side: revolutions per position of every rotary pair (double, and rounded to float for
  // the offsets inside a tile), and the angle of the first key of a tile (fraction of a revolution),
  // double-buffered like the stages
  __shared__ double rope_rate[ROPE_K ? D / 2 : 1];
  __shared__ __align__(16) float rope_rate_f[ROPE_K ? D / 2 : 4];
  __shared__ __align__(16) float rope_fr0[2][ROPE_K ? D / 2 : 4];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g2 = lane >> 5;
  const int Hq = p.n_q_heads, Hkv = p.n_kv_heads, r = p.rank;
  const int G = p.group;  // q heads whose rows share a q tile

  // workgroup -> (kv head, q tile); consecutive ids go to consecutive XCDs
  const int lin = blockIdx.x;
  const int rest = lin / Hkv, hk = lin - rest * Hkv;
  const int head_first = hk * G;
  // (the last tiles of a chunk see the most keys: they go first)
  const BatchTiles item = batch_tiles(p, static_cast<int>(gridDim.x) / Hkv - 1 - rest, lane);
  const int n_rows = item.n_queries * G;           // query rows of these heads: (new token, q head), the q head fastest
  const int t = item.t, a_idx = item.adapter, n_t = item.n_t;
  if (static_cast<int64_t>(item.tile) * BM >= n_rows) return;
  const int q0 = item.tile * BM;
  const int base_vis = item.first_pos;     // query i sees keys up to base_vis + i vis_step
  const int vis_step = p.causal ? 1 : 0;
  // First new token of the tile, how many of its q heads lie in the tile before, and the live rows of the tile.  A
  // lane's row is in_tile = 32 wave + l32 rows further: token tok0 + (head0 + in_tile) / G, the quotient (of at most
  // 143 by at most 16) taken exactly by a multiplication, so that it is cheap to form again wherever it is needed:
  // kept in registers through the loop it sent the rank-64 kernels to scratch memory (the three small numbers
  // travel in one scalar register for the same reason).
  const int tok0 = G > 1 ? __builtin_amdgcn_readfirstlane(q0 / G) : q0;
  const int row_map = (q0 - tok0 * G) | (min(BM, n_rows - q0) << 4) | (p.row_mul << 12);
  // (token - tok0, q head of the group) of a row of the tile; false (and the last live row) for one past the end
  auto map_row = [&](int in_tile, int& tok, int& gq) __attribute__((always_inline)) -> bool {
    int m = row_map;
    // (not at d = 64, rank 64 with a Qt term, where the kernel has registers left and, with this barrier to its
    // scheduling, walked a tile alone on its unit in 1.25 times the time)
    if constexpr (!(D == 64 && RP == 64 && HAS_BK)) asm volatile("" : "+s"(m), "+v"(in_tile));
    const int at = (m & 15) + min(in_tile, ((m >> 4) & 255) - 1);
    tok = (at * (m >> 12)) >> 16;
    gq = at - tok * G;
    return in_tile < ((m >> 4) & 255);
  };
  // index of this lane's row in q, out and the workspace; -1: a row past the end, never stored
  auto global_row = [&](bool clamped) __attribute__((always_inline)) -> int {
    int tok, gq;
    const bool live = map_row(wave * 32 + (static_cast<int>(threadIdx.x) & 31), tok, gq);
    return live || clamped ? (item.first_query + tok0 + tok) * Hq + head_first + gq : -1;
  };
  auto token_of = [&](int in_tile) __attribute__((always_inline)) -> int {
    int tok, gq;
    map_row(in_tile, tok, gq);
    return tok0 + tok;
  };
  auto limit_of = [&](int in_tile) __attribute__((always_inline)) -> int { return base_vis + vis_step * token_of(in_tile); };
  const int wave_first = __builtin_amdgcn_readfirstlane(limit_of(wave * 32));  // the smallest limit of this wave
  const int wave_last = __builtin_amdgcn_readfirstlane(limit_of(wave * 32 + 31));  // and the largest
  const int wg_last = __builtin_amdgcn_readfirstlane(limit_of(BM - 1));       // last key any row of the workgroup sees
  const bool live_wave = q0 + wave * 32 < n_rows;  // (a wave without rows helps with the tiles' traffic only)
  // (for the merge kernel, which keeps it inside the table)
  auto adapter_of = [&](int row) __attribute__((always_inline)) -> int {
    return vis_step != 0 || p.tile_per_query ? a_idx : p.query_adapter[row / Hq];
  };
  // Window: the first key that any row of the tile sees of its window, the sinks before it, and the key tiles between the
  // two that are passed over (tile number v of the workgroup is the sequence's tile v, or v + gap_tiles from sink_tiles on)
  int win_lo = 0, n_sinks = 0, sink_tiles = 0, gap_tiles = 0;
  if (p.window > 0) {
    win_lo = max(0, base_vis + vis_step * tok0 - p.window + 1);
    n_sinks = min(p.sinks, win_lo);
    sink_tiles = (n_sinks + BN - 1) / BN;
    gap_tiles = max(0, win_lo / BN - sink_tiles);
  }
  auto tile_key = [&](int tile) __attribute__((always_inline)) -> int {
    return (tile < sink_tiles ? tile : tile + gap_tiles) * BN;
  };
  const int n_tiles = wg_last < 0 ? 0 : wg_last / BN + 1 - gap_tiles;
  // this workgroup's share of the q tile's key tiles: [tile_begin, tile_end)
  const int split = SPLIT ? blockIdx.y : 0;
  const int tile_begin = SPLIT ? static_cast<int>(static_cast<int64_t>(n_tiles) * split / p.n_splits) : 0;
  const int tile_end = SPLIT ? static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / p.n_splits) : n_tiles;
  if constexpr (!SPLIT) {
    if (n_tiles == 0) {  // nothing is seen: zeros
      const int out_row = global_row(false);
      if (out_row >= 0)
        for (int c = g2 * 8; c < D; c += 16) *reinterpret_cast<uint4*>(static_cast<bf16_t*>(p.out) + static_cast<int64_t>(out_row) * D + c) = make_uint4(0u, 0u, 0u, 0u);
      return;
    }
  }
  if (SPLIT && tile_begin >= tile_end) {
    // more workgroups than key tiles: leave an empty state (zero row sum), all the merge
    // kernel looks at; for a row that sees nothing at all the first share leaves one that gives zeros
    const int out_row = global_row(false);
    if (out_row >= 0) {
      const int64_t slot = static_cast<int64_t>(out_row) * p.n_splits + split;
      const bool nothing = split == 0 && limit_of(wave * 32 + l32) < 0;
      if (g2 == 0) {
        p.part_ml[slot * 2 + 0] = nothing ? 0.f : -INFINITY;
        p.part_ml[slot * 2 + 1] = nothing ? 1.f : 0.f;
        if (split == 0) p.part_adapter[out_row] = adapter_of(out_row);
      }
      if (nothing) {
        for (int c = g2; c < D; c += 2) p.part_o[slot * D + c] = 0.f;
        for (int c = g2; c < r; c += 2) p.part_lr[slot * r + c] = 0.f;
      }
    }
    return;
  }

  // ---------------- tile traffic: HBM -> LDS, no registers in between ----------------
  const BatchTileLoader<D, RP, PAGED, POOL> loader(p, smem, wave, lane, hk, t, n_t, a_idx, n_sinks, win_lo);
  auto issue_tile = [&](int j, int st) { loader.issue_tile(j, st * STAGE); };

  if (PAGED) loader.fetch_ids(tile_key(tile_begin) / 16);
  issue_tile(tile_key(tile_begin), 0);
  if (ONES_ROW && tid == 0) *reinterpret_cast<pf_u32x4*>(smem + ONES_AT) = pf_u32x4{0x00003f80u, 0u, 0u, 0u};

  // ---------------- rotary key side: B_K^T operands of E^T, rotation rates ----------------
  // Wave (pair set ps = wave / 2, key half kt_e = wave % 2); d = 128: feature blocks ps and ps + 2,
  // d = 64: blocks 0 and 1 (waves 2, 3 have nothing to do).  A operand of E^T = B_K^T . L^T: lane
  // (feature l32 of the block, half g2), element e <-> rho = 16ks + 8(e/4) + 4g2 + e%4, the order in
  // which the L operand is read below.
  constexpr int E_WAVES = ROPE_K ? 2 * (D / 64) : 0;
  const int fb_lo = D == 128 ? (wave >> 1) : 0, fb_hi = D == 128 ? (wave >> 1) + 2 : 1;
  const int kt_e = wave & 1;
  pf_bf16x8 bkt[2][ROPE_K ? RKS : 1];
  if (ROPE_K) {
    if (tid < D / 2) {  // read after the barrier that precedes the loop
      const double rate = rope_rate_rev(tid, D, p.key_rope_theta);
      rope_rate[tid] = rate;
      rope_rate_f[tid] = static_cast<float>(rate);
      double rev = static_cast<double>(tile_key(tile_begin)) * rate;
      rev -= floor(rev);
      rope_fr0[0][tid] = static_cast<float>(rev);
    }
    if (wave < E_WAVES) {
      const int64_t ldb = static_cast<int64_t>(Hkv) * D;
      const bf16_t* bkg = static_cast<const bf16_t*>(p.b_k) + static_cast<int64_t>(a_idx) * r * ldb + hk * D;
#pragma unroll
      for (int sel = 0; sel < 2; ++sel)
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks) {
          uint32_t w4[4];
#pragma unroll
          for (int e2 = 0; e2 < 4; ++e2) {
            uint32_t pair = 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int e = 2 * e2 + x;
              const int rho = 16 * ks + 8 * (e >> 2) + 4 * g2 + (e & 3);
              const uint32_t v = rho < r ? bkg[rho * ldb + 32 * (sel == 0 ? fb_lo : fb_hi) + l32] : 0u;
              pair |= v << (16 * x);
            }
            w4[e2] = pair;
          }
          bkt[sel][ks] = pf_as_bf16x8(make_uint4(w4[0], w4[1], w4[2], w4[3]));
        }
    }
  }

  // ---------------- prologue: Q operands, Qt = Q B_K^T ----------------
  // qb[ks]: B operand of S^T: lane (row l32, k = 16ks + 8g2 + e)
  pf_bf16x8 qb[KS];
  {
    const bf16_t* qrow = static_cast<const bf16_t*>(p.q) + static_cast<int64_t>(global_row(true)) * D + g2 * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qb[ks] = pf_as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16));
  }
  pf_f16x8 qh[KF16 ? KS : 1];  // the same operands as fp16, for scores against fp16 keys
  if constexpr (KF16) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qh[ks] = pf_bf16x8_to_f16x8(qb[ks]);
  }
  // Qt^T[rho][row] = B_K[rho][:] . Q[row][:]: C layout lane (row l32; reg i <-> rho = 32b + 8(i/4) + 4g2 + i%4).
  // As B operand of the rank k-steps of S^T, k-step ks' takes registers 8ks'..8ks'+7 of
  // block b = ks'/2, i.e. element e <-> rho = 16ks' + 8(e/4) + 4g2 + e%4; the L operand
  // below is read in the same order.
  // Rows of several agents: one product per query of the wave's rows, kept in that query's lanes; the rows of B_K of the next
  // are requested before those of one are used.
  pf_bf16x8 qtb[RKS];
  if (HAS_BK) {
#pragma unroll
    for (int ks = 0; ks < RKS; ++ks) qtb[ks] = pf_as_bf16x8(make_uint4(0u, 0u, 0u, 0u));
    const int64_t ldb = static_cast<int64_t>(Hkv) * D;
    const bf16_t* bkg = static_cast<const bf16_t*>(p.b_k) + hk * D;
    const bool one = !SPLIT || vis_step != 0 || p.tile_per_query;  // adapter (rows of several leave states)
    const int tok_a = __builtin_amdgcn_readfirstlane(token_of(wave * 32)), tok_b = __builtin_amdgcn_readfirstlane(token_of(wave * 32 + 31));
    const int mine = token_of(wave * 32 + (static_cast<int>(threadIdx.x) & 31)) - tok_a;
    const int n_it = !SPLIT ? 1 : (!live_wave ? 0 : (one ? 1 : tok_b - tok_a + 1));
    pf_u32x4 bk[RB][KS];
    auto request = [&](int it) __attribute__((always_inline)) {
      const int a = one ? a_idx : min(max(__builtin_amdgcn_readfirstlane(p.query_adapter[item.first_query + tok_a + it]), 0), p.n_adapters - 1);
      // rows of this adapter's B_K for kv head hk; rows past the rank lie outside the resource and read as zero
      const __amdgpu_buffer_rsrc_t rs_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(bkg) + static_cast<int64_t>(a) * r * ldb, 0,
                                                                            static_cast<int>((static_cast<int64_t>(r - 1) * ldb + D) * 2), 0x00020000);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int rho = b * 32 + l32;
        const uint32_t boff = rho < r ? static_cast<uint32_t>(rho * ldb * 2 + g2 * 16) : kPfOob;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) bk[b][ks] = __builtin_amdgcn_raw_buffer_load_b128(rs_b, boff, ks * 32, 0);
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
        for (int ks = 0; ks < KS; ++ks)
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pf_bf16x8, bk[b][ks]), qb[ks], acc[b], 0, 0, 0);
      }
      if (it + 1 < n_it) request(it + 1);
      if (one || mine == it) {
#pragma unroll
        for (int ks2 = 0; ks2 < RKS; ++ks2) {
          const pf_f32x16& c = acc[ks2 >> 1];
          const int o = (ks2 & 1) * 8;
          qtb[ks2] = pf_as_bf16x8(make_uint4(pf_pack2(c[o + 0], c[o + 1]), pf_pack2(c[o + 2], c[o + 3]), pf_pack2(c[o + 4], c[o + 5]),
                                             pf_pack2(c[o + 6], c[o + 7])));
        }
      }
    }
  }

  // ---------------- per-lane LDS read offsets (stage 0; stage 1 is STAGE further) ----------------
  // K rows as A operand of S^T (ds_read_b128): key = 32kt + l32, logical chunk c = 2ks + g2
  // lives at chunk c ^ swizzle(key); row offset and swizzle occupy disjoint address bits,
  // so the address is k_pre ^ (c << 4) (+ kt * 32 rows)
  const int k_pre = l32 * (D * 2) + (pf_swz_k<D>(l32) << 4);
  // V^T as A operand of O^T (ds_read_b64_tr_b16): lane a of a 16-lane group addresses
  // row 4*g2 + a/4 (+ 8 for the second read) of the 16-key k-step, 8 bytes at
  // d = 32b + 16dsel + 4(a%4): chunk 4b + 2dsel + c0, half sub; the swizzle flips chunk
  // bits 2..3, so the address is v_pre ^ (b << 6) (+ row offsets)
  const int a16 = lane & 15;
  const int dsel = (lane >> 4) & 1;   // which 16 of the 32 output rows this 16-lane group produces
  const int vrow = 4 * g2 + (a16 >> 2);
  const int v_pre = K_BYTES + vrow * (D * 2) + ((((a16 & 3) >> 1) + 2 * dsel + pf_swz_v<D>(vrow)) << 4) + (a16 & 1) * 8;
  // L rows as A operand of S^T: two 8-byte pieces per k-step (chunks 2ks' and 2ks' + 1, half
  // g2); the swizzle of row 32kt + l32 does not depend on kt
  int l_rd[RKS][2];
#pragma unroll
  for (int ks = 0; ks < RKS; ++ks)
#pragma unroll
    for (int pc = 0; pc < 2; ++pc)
      l_rd[ks][pc] = 2 * K_BYTES + l32 * (RP * 2) + (((2 * ks + pc) ^ pf_swz_l<LCH>(l32)) << 4) + g2 * 8;
  // L^T as A operand of Olr^T: rows rho = 32b + 16dsel + 4(a%4) .. +3 of key vrow (+8 for the
  // second read; +16 per k-step does not change the swizzle).  In a half-empty last block
  // the upper 16 lanes read the constant [1, 0, 0, 0] instead: output row 32b + 16 then
  // accumulates the row sums; the rows after it are never used.
  int lt_rd[RB][2];
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int key = vrow + 8 * hh;
      const int ch = 4 * b + 2 * dsel + ((a16 & 3) >> 1);
      lt_rd[b][hh] = 2 * K_BYTES + key * (RP * 2) + (((ch & (LCH - 1)) ^ pf_swz_l<LCH>(key)) << 4) + (a16 & 1) * 8;
    }
  const bool ones_lane = ONES_ROW && dsel == 1;  // in block RB - 1

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
  // The running maximum is only raised when some row's tile maximum exceeds it by more than
  // kSlack (base-2 units): until then probabilities up to 2^kSlack are accumulated, which
  // fp32 sums and bf16 probabilities hold without loss, and the final division by the row
  // sum (taken with the same reference) cancels the factor exactly.
  constexpr float kSlack = 8.0f;
  constexpr int kReadAheadS = 8, kReadAheadPV = 6;

  pf_wait_vm0();
  __syncthreads();

  auto tile_step = [&](int tile, auto st_c) {
    constexpr int ST = decltype(st_c)::value;
    const int j = tile_key(tile);
    const unsigned char* ks_l = smem + ST * STAGE;  // K region; the V and L offsets are part of v_pre, l_rd, lt_rd
    const bool more = tile + 1 < tile_end;
    // the other stage was last read before the barrier that ended the previous tile; where
    // in the tile the requests are placed makes no measurable difference
    const int j_next = tile_key(tile + 1);
    if constexpr (PAGED) {
      if (more && j_next != j + BN) loader.fetch_ids(j_next / 16);  // (past the sinks: the ids at hand are of other blocks)
    }
    if (more) issue_tile(j_next, ST ^ 1);

    if (ROPE_K) {
      if (wave < E_WAVES) {
        pf_f32x16 e_lo, e_hi;
#pragma unroll
        for (int i = 0; i < 16; ++i) e_lo[i] = e_hi[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks) {
          const uint2 lo = *reinterpret_cast<const uint2*>(ks_l + l_rd[ks][0] + kt_e * 32 * RP * 2);
          const uint2 hi = *reinterpret_cast<const uint2*>(ks_l + l_rd[ks][1] + kt_e * 32 * RP * 2);
          const pf_bf16x8 lop = pf_as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y));
          e_lo = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bkt[0][ks], lop, e_lo, 0, 0, 0);
          e_hi = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bkt[1][ks], lop, e_hi, 0, 0, 0);
        }
        // register i of this lane: key 32 kt_e + l32 of the tile (position j + that), features
        // 32 fb + 8 (i/4) + 4 g2 + i%4 of blocks fb_lo, fb_hi: pair index = the fb_lo feature
        // Angle of (key, pair) in revolutions: that of the tile's first key, kept in double precision
        // by the table threads, plus the key's offset in the tile times the rate (at most 63 x 0.16
        // revolutions: single precision holds it to 1e-6).
        const int key = 32 * kt_e + l32;
        const float key_f = static_cast<float>(key);
        unsigned char* krow = smem + ST * STAGE + key * (D * 2) + 8 * g2;
        const int swz = pf_swz_k<D>(key);
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int dd0 = 32 * fb_lo + 8 * q4 + 4 * g2;
          const pf_f32x4 fr0 = *reinterpret_cast<const pf_f32x4*>(&rope_fr0[ST][dd0]);
          const pf_f32x4 rt = *reinterpret_cast<const pf_f32x4*>(&rope_rate_f[dd0]);
          float lo4[4], hi4[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * q4 + e;
            const float fr = fmaf(key_f, rt[e], fr0[e]);
            const float sn = __builtin_amdgcn_sinf(fr), cs = __builtin_amdgcn_cosf(fr);
            lo4[e] = e_lo[i] * cs - e_hi[i] * sn;
            hi4[e] = e_hi[i] * cs + e_lo[i] * sn;
          }
#pragma unroll
          for (int sel = 0; sel < 2; ++sel) {
            const float* add = sel == 0 ? lo4 : hi4;
            uint2* at = reinterpret_cast<uint2*>(krow + (((4 * (sel == 0 ? fb_lo : fb_hi) + q4) ^ swz) << 4));
            const uint2 old = *at;
            *at = make_uint2(pf_pack2_f16(__uint_as_float(old.x << 16) + add[0], __uint_as_float(old.x & 0xffff0000u) + add[1]),
                             pf_pack2_f16(__uint_as_float(old.y << 16) + add[2], __uint_as_float(old.y & 0xffff0000u) + add[3]));
          }
        }
      }
      __syncthreads();  // the completed keys are visible to the score loop of every wave
      if (more && tid < D / 2) {  // the next tile's first angle, for the expansion after the barrier that ends this tile
        double rev = static_cast<double>(j_next) * rope_rate[tid];
        rev -= floor(rev);
        rope_fr0[ST ^ 1][tid] = static_cast<float>(rev);
      }
    }

    if (SPLIT && !live_wave) {
      pf_wait_vm0();
      __syncthreads();
      return;
    }

    // S^T for the two 32-key halves of the tile.  The halves alternate, so consecutive
    // matrix instructions never wait for each other's result, and the LDS reads run
    // kReadAheadS operands ahead of the products that consume them.
    pf_f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const uint4 a4 = *reinterpret_cast<const uint4*>(ks_l + (k_pre ^ ((2 * ks + g2) << 4)) + kt * 32 * D * 2);
        if constexpr (KF16)
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(pf_f16x8, a4), qh[ks], s[kt], 0, 0, 0);
        else
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(a4), qb[ks], s[kt], 0, 0, 0);
      }
    if (HAS_BK) {
#pragma unroll
      for (int ks = 0; ks < RKS; ++ks)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const uint2 lo = *reinterpret_cast<const uint2*>(ks_l + l_rd[ks][0] + kt * 32 * RP * 2);
          const uint2 hi = *reinterpret_cast<const uint2*>(ks_l + l_rd[ks][1] + kt * 32 * RP * 2);
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y)), qtb[ks],
                                                          s[kt], 0, 0, 0);
        }
    }
    // instruction order for the scheduler: kReadAheadS LDS reads, then one product per read
    __builtin_amdgcn_sched_group_barrier(0x100, kReadAheadS, 0);
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if (HAS_BK) {
#pragma unroll
      for (int i = 0; i < 2 * RKS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
    }
    // causal mask + online softmax.  Element (kt, i) of this lane is key
    // j + 32kt + 8(i/4) + 4g2 + i%4 of row l32.
    if (j + BN - 1 > wave_first) {  // some row of this wave does not see the whole tile
      const int limit = limit_of(wave * 32 + (static_cast<int>(threadIdx.x) & 31));  // last visible key of this lane's row
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = j + 32 * kt + 8 * (i >> 2) + 4 * g2 + (i & 3);
          if (key > limit) s[kt][i] = -INFINITY;
        }
    }
    if (p.window > 0 && j + p.window <= wave_last && j + BN > p.sinks) {  // some row of this wave's window starts behind the first key
      const int first = limit_of(wave * 32 + (static_cast<int>(threadIdx.x) & 31)) - p.window + 1;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = j + 32 * kt + 8 * (i >> 2) + 4 * g2 + (i & 3);
          if (key < first && key >= p.sinks) s[kt][i] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
    mx = tile_reference(fmaxf(mx, pf_partner32(mx)) * sc);
    if (__builtin_amdgcn_ballot_w64(mx > m_run + kSlack) != 0) {  // always on the first tile (m_run = -inf)
      const float m_new = fmaxf(m_run, mx);
      // (a row may have seen nothing yet)
      const float alpha = (m_new == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int b = 0; b < DB; ++b) o_acc[b] *= alpha;
#pragma unroll
      for (int b = 0; b < RB; ++b) lr_acc[b] *= alpha;
    }
    const float nm = (m_run == -INFINITY) ? 0.f : -m_run;
    pf_bf16x8 pb[2][2];       // [kt][16-key k-step]
    auto exp_half = [&](int kt) __attribute__((always_inline)) {
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, nm));
        if (!ONES_ROW) l_run += e[i];
      }
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
        pb[kt][h2] = pf_as_bf16x8(make_uint4(pf_pack2(e[8 * h2 + 0], e[8 * h2 + 1]), pf_pack2(e[8 * h2 + 2], e[8 * h2 + 3]),
                                             pf_pack2(e[8 * h2 + 4], e[8 * h2 + 5]), pf_pack2(e[8 * h2 + 6], e[8 * h2 + 7])));
    };
    // The exponentials of the second 32-key half run under the products of the first: a matrix instruction
    // occupies its pipe for 32 cycles, and the wave is free to issue vector work meanwhile.
    exp_half(0);
    __builtin_amdgcn_sched_barrier(0);
    exp_half(1);
    // O^T += V^T P^T ; Olr^T += L^T P^T, one 16-key k-step at a time.
    // k-step (kt, h2), element e <-> key 32kt + 16h2 + 8(e/4) + 4g2 + e%4.
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        const int rowoff = (32 * kt + 16 * h2) * (D * 2);
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          const unsigned char* src = ks_l + (v_pre ^ (b << 6)) + rowoff;
          const pf_bf16x8 a = pf_join(pf_read_tr16(src), pf_read_tr16(src + 8 * (D * 2)));
          o_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[kt][h2], o_acc[b], 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const int koff = (32 * kt + 16 * h2) * (RP * 2);
          const unsigned char* src0 = ks_l + lt_rd[b][0] + koff;
          const unsigned char* src1 = ks_l + lt_rd[b][1] + koff;
          if (ONES_ROW && b == RB - 1) {
            src0 = ones_lane ? smem + ONES_AT : src0;
            src1 = ones_lane ? smem + ONES_AT : src1;
          }
          const pf_bf16x8 a = pf_join(pf_read_tr16(src0), pf_read_tr16(src1));
          lr_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[kt][h2], lr_acc[b], 0, 0, 0);
        }
      }
    // the transposed reads (two per operand) run kReadAheadPV operands ahead
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kReadAheadPV, 0);
#pragma unroll
    for (int i = 0; i < 2 * (DB + RB); ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, ONES_ROW ? 3 : 5, 0);
    }
#pragma unroll
    for (int i = 0; i < 2 * (DB + RB); ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    // the next tile has landed (this wave's share) and everybody is done reading this one
    pf_wait_vm0();
    __syncthreads();
  };
  for (int tile = tile_begin; tile < tile_end; tile += 2) {
    tile_step(tile, std::integral_constant<int, 0>{});
    if (tile + 1 < tile_end) tile_step(tile + 1, std::integral_constant<int, 1>{});
  }

  // ---------------- epilogue: O^T += B_V^T Olr^T, O /= l, store ----------------
  const int out_row = global_row(false);
  if (ONES_ROW) {
    // row sums sit in register 8 (rho = 32(RB-1) + 16) of the lanes with g2 == 0
    const float mine = lr_acc[RB - 1][8];
    const float other = pf_partner32(mine);
    l_run = g2 == 0 ? mine : other;
  } else {
    l_run += pf_partner32(l_run);
  }
  if (SPLIT) {
    // this share's state for the merge kernel: m in natural-log units, l, O^T and Olr^T as
    // fp32 rows [slot][d] and [slot][rank]; registers 4q..4q+3 are d (rho) = 32b + 8q + 4g2 + 0..3
    if (out_row >= 0) {
      const int64_t slot = static_cast<int64_t>(out_row) * p.n_splits + split;
      if (g2 == 0) {
        const bool nothing = split == 0 && limit_of(wave * 32 + l32) < 0;  // (such a row's O and O_lr are zeros)
        p.part_ml[slot * 2 + 0] = nothing ? 0.f : m_run * 0.69314718055994530942f;
        p.part_ml[slot * 2 + 1] = nothing ? 1.f : l_run;
        if (split == 0) p.part_adapter[out_row] = adapter_of(out_row);
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
    return;
  }
  if (p.b_v != nullptr) {
    const int64_t ldb = static_cast<int64_t>(Hkv) * D;
    const bf16_t* bv = static_cast<const bf16_t*>(p.b_v) + static_cast<int64_t>(a_idx) * r * ldb + hk * D;
#pragma unroll
    for (int ks = 0; ks < RKS; ++ks) {
      // B operand: Olr^T registers 8(ks&1)..+7 of block ks/2: element e <-> rho = 16ks + 8(e/4) + 4g2 + e%4
      const int o = (ks & 1) * 8;
      const pf_f32x16& src = lr_acc[ks >> 1];
      // O_lr as two bf16 terms, the second what the first left over: to 17 bits, against the 8 of the output's own
      // rounding.  (One term cost up to 2^-9 of |O_lr| |B_V|, which calls with several shares, whose merge holds
      // O_lr in fp32, do not pay; 32 to 64 cycles of matrix pipe per 16 ranks and 32 columns, once per q tile.)
      pf_bf16x8 bop[2];
      {
        uint32_t w[2][4];
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) {
          const float x0 = src[o + 2 * e2], x1 = src[o + 2 * e2 + 1];
          w[0][e2] = pf_pack2(x0, x1);
          const float r0 = x0 - __uint_as_float(w[0][e2] << 16), r1 = x1 - __uint_as_float(w[0][e2] & 0xffff0000u);
          w[1][e2] = pf_pack2(__builtin_isfinite(r0) ? r0 : 0.f, __builtin_isfinite(r1) ? r1 : 0.f);
        }
#pragma unroll
        for (int term = 0; term < 2; ++term) bop[term] = pf_as_bf16x8(make_uint4(w[term][0], w[term][1], w[term][2], w[term][3]));
      }
      pf_bf16x8 bvt[DB];
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        // A operand: B_V^T: lane (d = 32b + l32, element e <-> rho as above)
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int rho = 16 * ks + 8 * (e >> 2) + 4 * g2 + (e & 3);
          const uint32_t val = rho < r ? static_cast<uint32_t>(bv[rho * ldb + 32 * b + l32]) : 0u;
          w[e >> 1] |= val << ((e & 1) * 16);
        }
        bvt[b] = pf_as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
      }
#pragma unroll
      for (int term = 1; term >= 0; --term)
#pragma unroll
        for (int b = 0; b < DB; ++b) o_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bvt[b], bop[term], o_acc[b], 0, 0, 0);
    }
  }
  if (out_row >= 0) {
    const float inv = limit_of(wave * 32 + l32) < 0 ? 0.f : 1.0f / l_run;  // (a row that sees nothing: zeros)
    bf16_t* orow = static_cast<bf16_t*>(p.out) + static_cast<int64_t>(out_row) * D;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // registers 4q..4q+3 are d = 32b + 8q + 4g2 + 0..3
        const uint2 pk = make_uint2(pf_pack2(o_acc[b][4 * q + 0] * inv, o_acc[b][4 * q + 1] * inv),
                                    pf_pack2(o_acc[b][4 * q + 2] * inv, o_acc[b][4 * q + 3] * inv));
        *reinterpret_cast<uint2*>(orow + 32 * b + 8 * q + 4 * g2) = pk;
      }
  }
}

template <int D, int RP, bool PAGED, bool POOL, bool HAS_BK, bool SPLIT, bool ROPE_K>
__global__ __launch_bounds__(256, 2) void batch_tiles_kernel(BatchParams p) {
  batch_tiles_body<D, RP, PAGED, POOL, HAS_BK, SPLIT, ROPE_K>(p);
}

}  // namespace lra
