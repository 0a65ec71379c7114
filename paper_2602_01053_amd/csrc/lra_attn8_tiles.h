// Tile-walking attention over 8-bit codes (bf16, gfx950): chunks of new tokens of many sequences, and more agents than the few-rows
// kernel takes.  The tile, its mapping to sequences, masks and epilogue are those of batch_tiles_kernel (lra_batch_tiles.h), with one
// low-rank cache and no rotated key side; what differs is how K and V come to LDS.
//
// The codes of the next tile travel through registers, 64 bytes a thread, and are written to the other stage as bf16 once the products
// of this one are done: each code is converted once for the 128 rows of the tile, not once per wave.  They are written in the order in
// which the products read them, a KB per instruction's operand:
//   K: k-step ks of 32 keys is the rows' chunk ks, key l32 in slot l32 + 32 g2; the slots of a chunk are exchanged in pairs (xor) so
//      that eight lanes holding the chunks of one row do not meet in a bank;
//   V: the cache holds sixteen tokens of a dimension together, which are two lanes' operands of O^T += V^T P^T: tokens 0-3 and 8-11,
//      4-7 and 12-15, as the score registers have them.  No transposed reads (batch_tiles_kernel takes two per operand).
// Bound by what a step of 64 keys issues: chunks of 2048 and 1376 tokens over 18 k and 13 k take 1055 us, 0.93 PFLOP/s (matrix cores busy
// 41 %, vector units and LDS 38 % each; two workgroups to a compute unit); the same call on 16-bit rows takes 1016, without the conversion.
#pragma once

#include "lra_attn8_rows.h"

namespace lra {

// Workgroup `at` -> q tile, those that see the most tokens first (in classes of 256 of them), so that none of those begins when the others are
// done: 32 chunks of unlike contexts take a fifth less.  Every workgroup finds its tile by itself: a class by bisection over the number of tiles from a class on, which
// for a sequence's tiles, each seeing more than the one before, is a quotient; then the sequence by a running sum over its class.
__device__ __forceinline__ bool attn8_longest_first(const Batch8Params& p, int at, int lane, BatchTiles& item) {
  constexpr int N = kShareSeqs / 64;
  int tiles[N], first_pos[N], new_tokens[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Attn8Sequence s = attn8_sequence(p, min(64 * i + lane, p.n_seqs - 1));
    new_tokens[i] = 64 * i + lane < p.n_seqs ? s.c1 - s.c0 : 0;  // (none, and no tiles of any class, behind the last)
    tiles[i] = (new_tokens[i] * p.group + 127) >> 7;
    first_pos[i] = s.first_pos;
  }
  // the first of sequence i's tiles of class `cls` and above
  auto first_of = [&](int i, int cls) __attribute__((always_inline)) -> int {
    if (cls <= 0) return 0;
    if (p.window > 0 && cls * 256 > p.window + p.sinks) return tiles[i];  // (that many tokens nobody sees)
    const int x = cls * 256 - 1 - first_pos[i];
    return x <= 0 ? 0 : (!p.causal || x >= new_tokens[i] ? tiles[i] : (x * p.group) >> 7);
  };
  auto count = [&](int cls) __attribute__((always_inline)) -> int {
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c += tiles[i] - first_of(i, cls);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) c += __shfl_xor(c, off, kWave);
    return __builtin_amdgcn_readfirstlane(c);
  };
  if (at >= count(0)) return false;
  int cls = 0, beyond = (p.max_seq_len >> 8) + 1;  // count(cls) > at >= count(beyond) = 0
  while (beyond - cls > 1) {
    const int mid = (cls + beyond) >> 1;
    if (count(mid) > at) cls = mid;
    else beyond = mid;
  }
  at -= count(cls + 1);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int end = first_of(i, cls + 1), mine = end - first_of(i, cls);
    int upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int below = __shfl_up(upto, off, kWave);
      upto += lane >= off ? below : 0;
    }
    const uint64_t there = __builtin_amdgcn_ballot_w64(at < upto);
    if (there != 0) {
      const int k = __builtin_ctzll(there);
      item.t = 64 * i + k;
      item.tile = __builtin_amdgcn_readlane(end, k) - 1 - (at - (__builtin_amdgcn_readlane(upto, k) - __builtin_amdgcn_readlane(mine, k)));
      const Attn8Sequence s = attn8_sequence(p, item.t);
      item.n_t = __builtin_amdgcn_readfirstlane(s.n_t);
      item.first_query = __builtin_amdgcn_readfirstlane(s.c0);
      item.n_queries = __builtin_amdgcn_readfirstlane(s.c1 - s.c0);
      item.first_pos = __builtin_amdgcn_readfirstlane(s.first_pos);
      item.adapter = __builtin_amdgcn_readfirstlane(min(max(p.query_adapter[s.c0], 0), p.n_adapters - 1));
      return true;
    }
    at -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// Key tiles of a share, where the q tiles of several sequences (kShareSeqs at most) are shared out by their lengths: about head_shares
// shares of a kv head in all.
__device__ __forceinline__ int attn8_tiles_per_share(const Batch8Params& p, int lane) {
  float steps = 0.f;
#pragma unroll
  for (int i = 0; i < kShareSeqs / 64; ++i) {
    const Attn8Sequence s = attn8_sequence(p, min(64 * i + lane, p.n_seqs - 1));
    const int q_tiles = ((s.c1 - s.c0) * p.group + 127) >> 7;
    steps += 64 * i + lane < p.n_seqs ? static_cast<float>(s.n_tiles) * static_cast<float>(q_tiles) : 0.f;
  }
  steps = wave_sum(steps);
  return __builtin_amdgcn_readfirstlane(max(2, static_cast<int>(fminf(ceilf(steps / static_cast<float>(p.head_shares)), 1e9f))));
}

// A thread's codes and low-rank elements of one tile.
template <int D, int RP>
struct Attn8Pieces {
  static constexpr int N = D / 64;  // 16-byte pieces of K, and of V
  uint4 k[N], v[N], l;              // of L: rank 16 only, the first two waves
  int ks[N], vs[N];  // their scales
};

template <int D, int RP, int CODE>
struct Attn8Loader {
  static constexpr int BN = 64, KCH = D / 16, KS = D / 16, DB = D / 32;  // (chunks of sixteen dimensions per K row)
  static constexpr int K_BYTES = BN * D * 2;
  static constexpr int LCH = RP / 8, LROWS = 64 / LCH;  // 16-byte chunks of an L row, rows that a wave moves at once
  static constexpr int N = Attn8Pieces<D, RP>::N;

  const Batch8Params& p;
  unsigned char* const smem;
  uint32_t lds0;
  int wave, lane, h, seq, n_t, nb_last, cut_lo, cut_hi;
  mutable int ids = 0;  // block ids of an aligned group of 64 blocks, lane l holding that of block l of the group

  static __device__ __forceinline__ constexpr int swizzle(int ks) { return (KCH == 8 ? 2 * ks : 4 * ks) << 4; }
  __device__ __forceinline__ bool kept(int tok) const { return tok < n_t && (tok < cut_lo || tok >= cut_hi); }
  __device__ __forceinline__ bool whole(int j) const { return j + BN <= n_t && (j + BN <= cut_lo || j >= cut_hi); }
  // (blocks that hold no token that is seen may have any id: the one of the sequence's last stands in, whose codes are then zeroed)
  __device__ __forceinline__ void fetch_ids(int b) const {
    const int at = min((b & ~63) + lane, nb_last);
    const bool any = at * 16 < cut_lo || at * 16 + 15 >= cut_hi;
    ids = block8(p.block_table, p.max_blocks_per_seq, seq, any ? at : nb_last);
  }
  __device__ __forceinline__ int block_id(int b) const { return __builtin_amdgcn_readlane(ids, b & 63); }

  __device__ __forceinline__ Attn8Loader(const Batch8Params& p_, unsigned char* smem_, int wave_, int lane_, int h_, int t, int n_t_, int cut_lo_, int cut_hi_)
      : p(p_), smem(smem_), wave(wave_), lane(lane_), h(h_), seq(t), n_t(n_t_), cut_lo(cut_lo_), cut_hi(cut_hi_) {
    nb_last = (n_t - 1) >> 4;
    lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem)));
  }
  // block of the tile that piece i of this wave comes from
  __device__ __forceinline__ int block_of(int i) const { return D == 128 ? 2 * i + (wave >> 1) : wave; }

  // (an address that the whole wave shares, and the lane's offset in 32 bits)
  __device__ __forceinline__ uint4 piece(const void* codes, int64_t id) const {
    const uint8_t* base = static_cast<const uint8_t*>(codes) + id * p.kv_block_stride + h * p.kv_head_stride + (D == 128 ? (wave & 1) * 1024 : 0);
    return *reinterpret_cast<const uint4*>(base + static_cast<uint32_t>(lane * 16));
  }

  // the tile at key j into registers: K and L, then V, whose request asks for the next block ids as well
  __device__ __forceinline__ void request_kl(int j, uint32_t stage_off, Attn8Pieces<D, RP>& raw) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t id = block_id((j >> 4) + block_of(i));
      raw.k[i] = piece(p.k_base, id);
      raw.ks[i] = p.k_scale[id * p.scale_block_stride + h];
    }
    // L rows that nobody sees read as zeros.  A wave's sixteen rows or fewer lie in one block: straight into LDS, a resource per block;
    // at rank 16 two waves have thirty-two of two blocks each, through registers.
    if constexpr (LROWS > 16) {
      const int row = wave * LROWS + lane / LCH, c = lane % LCH;
      raw.l = make_uint4(0u, 0u, 0u, 0u);
      if (wave * LROWS < BN && kept(j + row) && c * 8 < p.rank) {
        const int b0 = (j + wave * LROWS) >> 4;
        const int64_t id = lane < 32 ? block_id(b0) : block_id(b0 + 1);
        raw.l = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(p.l) + (id * 16 + (row & 15)) * p.l_row_stride + c * 8);
      }
    } else {
      const uint32_t lp2 = static_cast<uint32_t>(p.l_row_stride) * 2u;  // (strides up to 2^24 elements)
#pragma unroll
      for (int q = 0; q < LCH / 4; ++q) {
        const int i = wave + 4 * q, tok0 = j + i * LROWS, row = i * LROWS + lane / LCH;
        const int c = (lane % LCH) ^ pf_swz_l<LCH>(row);
        const bf16_t* base = static_cast<const bf16_t*>(p.l) + static_cast<int64_t>(block_id(tok0 >> 4)) * 16 * p.l_row_stride;
        const uint32_t off = kept(j + row) && c * 8 < p.rank ? static_cast<uint32_t>((j + row) & 15) * lp2 + (c << 4) : kPfOob;
        pf_load16_to_lds(pf_rsrc(base, 15u * lp2 + static_cast<uint32_t>(p.rank) * 2u), lds0 + stage_off + 2 * K_BYTES + i * 1024, off, 0);
      }
    }
  }
  __device__ __forceinline__ void request_v(int j, Attn8Pieces<D, RP>& raw) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t id = block_id((j >> 4) + block_of(i));
      raw.v[i] = piece(p.v_base, id);
      raw.vs[i] = p.v_scale[id * p.scale_block_stride + h];
    }
    // the ids of the next sixteen tiles travel behind the requests of the last of this sixteen
    if ((((j >> 4) + 4) & 63) == 0) fetch_ids((j >> 4) + 4);
  }
  // the codes as bf16 values, and the L rows, into the stage at stage_off
  __device__ __forceinline__ void convert_kl(uint32_t stage_off, const Attn8Pieces<D, RP>& raw) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float ks = scale8(__builtin_amdgcn_readfirstlane(raw.ks[i]));
      const int blk = block_of(i);
      {
        const uint4 lo = codes_to_values<CODE>(raw.k[i].x, raw.k[i].y, ks), hi = codes_to_values<CODE>(raw.k[i].z, raw.k[i].w, ks);
        const int key = 16 * blk + (D == 128 ? (wave & 1) * 8 + (lane >> 3) : lane >> 2), c = lane % KCH;
        unsigned char* dst = smem + stage_off + ((key >> 5) * KS + c) * 1024;
        const int slot = ((key & 31) << 4) ^ swizzle(c);
        *reinterpret_cast<uint4*>(dst + (slot & 511)) = lo;
        *reinterpret_cast<uint4*>(dst + 512 + (slot & 511)) = hi;
      }
    }
    // (L rows: dense, chunks swizzled as the reads of both products have it)
    if constexpr (LROWS > 16) {
      const int row = wave * LROWS + lane / LCH, c = lane % LCH;
      if (wave * LROWS < BN) *reinterpret_cast<uint4*>(smem + stage_off + 2 * K_BYTES + row * (RP * 2) + ((c ^ pf_swz_l<LCH>(row)) << 4)) = raw.l;
    }
  }
  __device__ __forceinline__ void convert_v(int j, uint32_t stage_off, const Attn8Pieces<D, RP>& raw) const {
    const bool all = whole(j);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float vs = scale8(__builtin_amdgcn_readfirstlane(raw.vs[i]));
      const int blk = block_of(i);
      uint4 v = raw.v[i];
      if (!all) v = masked(v, token_masks(j + 16 * blk, n_t, cut_lo, cut_hi));  // tokens that nobody sees: their codes may be no numbers
      const uint4 lo = codes_to_values<CODE>(v.x, v.y, vs), hi = codes_to_values<CODE>(v.z, v.w, vs);
      const int d = (D == 128 ? (wave & 1) * 64 : 0) + lane;
      unsigned char* dst = smem + stage_off + K_BYTES + (blk * DB + (d >> 5)) * 1024 + ((d & 31) << 4);
      *reinterpret_cast<uint4*>(dst) = make_uint4(lo.x, lo.y, hi.x, hi.y);        // tokens 0-3, 8-11
      *reinterpret_cast<uint4*>(dst + 512) = make_uint4(lo.z, lo.w, hi.z, hi.w);  // tokens 4-7, 12-15
    }
  }
};

template <int D, int RP, bool HAS_BK, bool SPLIT, int CODE>
__global__ __launch_bounds__(256, 2) void attn8_tiles_kernel(Batch8Params p) {
  constexpr int BM = 128, BN = 64;
  // d = 128 and ranks above 32: K and L of the next tile go to LDS behind the scores, where V's codes are asked for (all held to the
  // end of the tile, the kernel went to scratch memory)
  constexpr bool K_EARLY = D == 128 && RP == 64;
  constexpr int KS = D / 16;   // k-steps of S^T over the head dimension
  constexpr int RKS = RP / 16; // k-steps over the padded rank
  constexpr int DB = D / 32;   // 32-row blocks of O^T
  constexpr int RB = (RP + 31) / 32;  // 32-row blocks of Olr^T
  constexpr int LCH = RP / 8;         // 16-byte chunks per L row (2, 4 or 8)
  constexpr int K_BYTES = BN * D * 2;
  constexpr int L_BYTES = BN * RP * 2;
  constexpr int STAGE = 2 * K_BYTES + L_BYTES;
  // With a half-empty last 32-row block of Olr^T (rank 16 or 48 after padding), its idle
  // upper lanes read a constant [1, 0, 0, 0] instead of L, so the matrix core also
  // accumulates the softmax row sums, of the probabilities as they are rounded to bf16: what O is divided by are the weights that
  // it was summed with.
  constexpr bool ONES_ROW = (RP % 32) != 0;
  constexpr int ONES_AT = 2 * STAGE;

  __shared__ __align__(16) unsigned char smem[2 * STAGE + (ONES_ROW ? 16 : 0)];
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
  // (the last tiles of a chunk see the most keys: they go first, of several chunks the longest of all)
  BatchTiles item;
  if (p.longest_first) {
    if (!attn8_longest_first(p, rest, lane, item)) return;
  } else {
    item = batch_tiles(p, static_cast<int>(gridDim.x) / Hkv - 1 - rest, lane);
  }
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
    return vis_step != 0 ? a_idx : p.query_adapter[row / Hq];
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
  int shares = p.n_splits;
  if (SPLIT && p.head_shares > 0) {
    const int per = max(attn8_tiles_per_share(p, lane), (n_tiles + p.n_splits - 1) / p.n_splits);
    shares = __builtin_amdgcn_readfirstlane(max(1, (n_tiles + per - 1) / per));
  }
  const int tile_begin = SPLIT ? (split < shares ? static_cast<int>(static_cast<int64_t>(n_tiles) * split / shares) : n_tiles) : 0;
  const int tile_end = SPLIT ? (split < shares ? static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / shares) : n_tiles) : n_tiles;
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

  // ---------------- tile traffic ----------------
  const Attn8Loader<D, RP, CODE> loader(p, smem, wave, lane, hk, t, n_t, n_sinks, win_lo);
  Attn8Pieces<D, RP> raw;  // codes on their way
  loader.fetch_ids(tile_key(tile_begin) / 16);
  auto request_first = [&]() __attribute__((always_inline)) {
    loader.request_kl(tile_key(tile_begin), 0, raw);
    loader.request_v(tile_key(tile_begin), raw);
  };
  if (!K_EARLY) request_first();
  if (ONES_ROW && tid == 0) *reinterpret_cast<pf_u32x4*>(smem + ONES_AT) = pf_u32x4{0x00003f80u, 0u, 0u, 0u};

  // ---------------- prologue: Q operands, Qt = Q B_K^T ----------------
  // qb[ks]: B operand of S^T: lane (row l32, k = 16ks + 8g2 + e)
  pf_bf16x8 qb[KS];
  {
    const bf16_t* qrow = static_cast<const bf16_t*>(p.q) + static_cast<int64_t>(global_row(true)) * D + g2 * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qb[ks] = pf_as_bf16x8(*reinterpret_cast<const uint4*>(qrow + ks * 16));
  }
  // (in bf16, as in attn8_rows_kernel)
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
    const bool one = !SPLIT || vis_step != 0;  // adapter (rows of several leave states)
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

  if (K_EARLY) request_first();  // (before, its registers met those of the rows of B_K)

  // ---------------- per-lane LDS read offsets (stage 0; stage 1 is STAGE further) ----------------
  // K as A operand of S^T: k-step (kt, ks) is a KB of its own, its slots exchanged as the writer did
  const int k_pre = lane << 4;
  // V^T as A operand of O^T: (kt, h2, b) likewise, as it lies
  const int v_pre = K_BYTES + (lane << 4);
  const int a16 = lane & 15;
  const int dsel = (lane >> 4) & 1;   // which 16 of the 32 output rows this 16-lane group produces
  const int vrow = 4 * g2 + (a16 >> 2);
  // L rows as A operand of S^T: two 8-byte pieces per k-step (chunks 2ks' and 2ks' + 1, half
  // g2); the swizzle of row 32kt + l32 does not depend on kt
  // (chunk c at l_pre ^ (c << 4): row offset, half and chunk occupy disjoint address bits)
  const int l_pre = 2 * K_BYTES + l32 * (RP * 2) + (pf_swz_l<LCH>(l32) << 4) + g2 * 8;
  // L^T as A operand of Olr^T: rows rho = 32b + 16dsel + 4(a%4) .. +3 of key vrow (+8 for the
  // second read; +16 per k-step does not change the swizzle).  In a half-empty last block
  // the upper 16 lanes read the constant [1, 0, 0, 0] instead: output row 32b + 16 then
  // accumulates the row sums; the rows after it are never used.
  // (block b and half hh at lt_pre, exclusive or the bits in which their chunk and swizzle differ, hh eight rows further)
  constexpr int LT_HALF = LCH == 8 ? 64 : (LCH == 4 ? 32 : 16);
  static_assert(RP != 16 || RB == 1);
  const int lt_pre = 2 * K_BYTES + vrow * (RP * 2) + (((((a16 & 3) >> 1) + 2 * dsel) & (LCH - 1)) << 4 ^ pf_swz_l<LCH>(vrow) << 4) + (a16 & 1) * 8;
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
  constexpr int kReadAheadS = K_EARLY ? 6 : 8, kReadAheadPV = K_EARLY ? 3 : 6;

  loader.convert_kl(0, raw);
  loader.convert_v(tile_key(tile_begin), 0, raw);
  if (RP > 16) pf_wait_vm0();  // (L, which the compiler does not know of)
  __syncthreads();

  auto tile_step = [&](int tile, auto st_c) {
    constexpr int ST = decltype(st_c)::value;
    const int j = tile_key(tile);
    const unsigned char* ks_l = smem + ST * STAGE;  // K region; the V and L offsets are part of v_pre, l_rd, lt_rd
    const bool more = tile + 1 < tile_end;
    // (the other stage was last read before the barrier that ended the previous tile)
    const int j_next = tile_key(tile + 1);
    if (more) {
      if (j_next != j + BN) loader.fetch_ids(j_next / 16);  // (past the sinks: the ids at hand are of other blocks)
      loader.request_kl(j_next, (ST ^ 1) * STAGE, raw);
      if (!K_EARLY || (SPLIT && !live_wave)) loader.request_v(j_next, raw);
    }

    if (SPLIT && !live_wave) {
      if (more) {
        loader.convert_kl((ST ^ 1) * STAGE, raw);
        loader.convert_v(j_next, (ST ^ 1) * STAGE, raw);
      }
      if (RP > 16) pf_wait_vm0();
      __syncthreads();
      return;
    }

    // S^T for the two 32-key halves of the tile.  The halves alternate, so consecutive
    // matrix instructions never wait for each other's result, and the LDS reads run
    // kReadAheadS operands ahead of the products that consume them.  The wave goes ahead of the SIMD's other one meanwhile
    // and, before all, while it converts the next tile, which three other waves wait for; softmax and V's products are what goes on beside:
    // chunks of 2048 and 1376 tokens over 18 k and 13 k take 1055 us, 1105 without, 1090 with the scores alone or V's products too.
    __builtin_amdgcn_s_setprio(1);
    pf_f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const uint4 a4 = *reinterpret_cast<const uint4*>(ks_l + (k_pre ^ Attn8Loader<D, RP, CODE>::swizzle(ks)) + (kt * KS + ks) * 1024);
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pf_as_bf16x8(a4), qb[ks], s[kt], 0, 0, 0);
      }
    if (HAS_BK) {
      int l_at = l_pre;
      if constexpr (RP > 16) asm volatile("" : "+v"(l_at));  // (addresses formed again for each tile: held in registers they went to scratch memory)
#pragma unroll
      for (int ks = 0; ks < RKS; ++ks)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const uint2 lo = *reinterpret_cast<const uint2*>(ks_l + (l_at ^ ((2 * ks) << 4)) + kt * 32 * RP * 2);
          const uint2 hi = *reinterpret_cast<const uint2*>(ks_l + (l_at ^ ((2 * ks + 1) << 4)) + kt * 32 * RP * 2);
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
    __builtin_amdgcn_s_setprio(0);
    if (K_EARLY && more) {
      __builtin_amdgcn_sched_barrier(0);
      loader.convert_kl((ST ^ 1) * STAGE, raw);
      __builtin_amdgcn_sched_barrier(0);
      loader.request_v(j_next, raw);
      __builtin_amdgcn_sched_barrier(0);
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
    int lt_at = lt_pre;
    if constexpr (RP > 16) asm volatile("" : "+v"(lt_at));  // (as l_at)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          const pf_bf16x8 a = pf_as_bf16x8(*reinterpret_cast<const uint4*>(ks_l + v_pre + ((2 * kt + h2) * DB + b) * 1024));
          o_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[kt][h2], o_acc[b], 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const int koff = (32 * kt + 16 * h2) * (RP * 2);
          const unsigned char* src0 = ks_l + (lt_at ^ (b << 6)) + koff;
          const unsigned char* src1 = ks_l + (lt_at ^ (b << 6) ^ LT_HALF) + 8 * (RP * 2) + koff;
          if (ONES_ROW && b == RB - 1) {
            src0 = ones_lane ? smem + ONES_AT : src0;
            src1 = ones_lane ? smem + ONES_AT : src1;
          }
          const pf_bf16x8 a = pf_join(pf_read_tr16(src0), pf_read_tr16(src1));
          lr_acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[kt][h2], lr_acc[b], 0, 0, 0);
        }
      }
    // the reads (one per operand of V, two of L) run kReadAheadPV ahead
    __builtin_amdgcn_sched_group_barrier(0x100, kReadAheadPV, 0);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, ONES_ROW ? 3 : 5, 0);
      }
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, ONES_ROW ? 3 : 5, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
    }
    __builtin_amdgcn_s_setprio(2);
    if (more) {
      if (!K_EARLY) loader.convert_kl((ST ^ 1) * STAGE, raw);
      loader.convert_v(j_next, (ST ^ 1) * STAGE, raw);
    }
    // the next tile has landed (this wave's share) and everybody is done reading this one
    if (RP > 16) pf_wait_vm0();
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

template <int D, int CODE>
static hipError_t launch_attn8_tiles(const Batch8Params& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.tile_places * p.n_kv_heads), p.n_splits);
  auto launch = [&](auto rp_c, auto split_c) {
    constexpr int RP = decltype(rp_c)::value;
    constexpr bool SPLIT = decltype(split_c)::value || (D == 128 && RP == 64);  // (the plan gives those states whatever the shares)
    if (p.b_k != nullptr) hipLaunchKernelGGL((attn8_tiles_kernel<D, RP, true, SPLIT, CODE>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attn8_tiles_kernel<D, RP, false, SPLIT, CODE>), grid, dim3(256), 0, s, p);
  };
  auto by_rank = [&](auto split_c) {
    if (p.rank <= 16) launch(std::integral_constant<int, 16>{}, split_c);
    else if (p.rank <= 32) launch(std::integral_constant<int, 32>{}, split_c);
    else launch(std::integral_constant<int, 64>{}, split_c);
  };
  if (p.part_ml != nullptr) by_rank(std::true_type{});
  else by_rank(std::false_type{});
  return hipGetLastError();
}

}  // namespace lra
