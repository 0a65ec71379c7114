// Attention over 8-bit codes for sequences with few query rows (bf16, gfx950): 16 at most per kv head, a decode step of some
// agents or a few tokens, through a window and sinks or not.
//
// One workgroup streams a share of one (sequence, kv head)'s visible keys for all its rows; its four waves take 64-key tiles in turn,
// four blocks each, and are on their own from the first tile to the last:
//   S^T = K Q^T + L Qt^T,   online softmax along keys,   O^T += V^T P^T,   Olr^T += L^T P^T      (v_mfma_f32_16x16x32_bf16)
// Nothing passes through LDS on the way: the layout of the cache is that of the operands.  Which key stands in which row of a product
// is free, as long as the next product agrees, and so is the order of the dimension that a product sums over:
//   row rho of key tile t (of four) is token 4t + rho % 4 of block rho / 4.  A lane of the A operand then takes 16 bytes
//     of every 64 of one token's K row, with Q's dimensions in the same order: a load's four lanes of a row have 64 bytes in a piece;
//   lane group g of the result S^T holds all sixteen tokens of block g, which is what the B operand of V^T P^T wants of it: its A
//     operand is sixteen tokens of one dimension, the 16 bytes that the cache holds together;
//   L is transposed by a product with the identity: the result layout of L I is the operand layout of L^T.
// A code becomes bf16 with its block's scale in one instruction per pair (e4m3) or by itself (integers, whose scores take K's scale and whose
// weights V's over a unit, powers of two both): the codes of a tile cost a wave some 500 cycles, the 16 KB that they stand for 2000 of the memory's.
// K of a wave's next tile is requested as soon as its scores are taken, V and L as soon as the products are: with eight waves to a
// compute unit some hundred KB are on their way.
// Bound by HBM where the shares are long: 14 rows over 16 sequences of 4 k to 64 k tokens 141 us with the merge, 5.5 TB/s of the bytes
// needed (a large copy reaches 5.2, both directions counted); 16 rows over 32 k tokens of 8 kv heads 17.5 us (68 MB), of which the start, two dependent round trips and Q B_K^T, is 5.
#pragma once

#include "lra_attn8_plan.h"
#include "lra_codes.h"
#include "lra_decode_util.h"

namespace lra {

typedef short s16x4v __attribute__((ext_vector_type(4)));

// Eight codes (two words) as bf16, times a power of two where CODE is e4m3.
template <int CODE>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  uint32_t o[4];
  if constexpr (CODE == LRA_E4M3) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  } else {
    // (integers of up to eight bits: exact in the upper half of a float)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = i < 2 ? lo : hi;
      const float a = static_cast<float>(static_cast<signed char>(w >> (16 * (i & 1)))), b = static_cast<float>(static_cast<signed char>(w >> (16 * (i & 1) + 8)));
      o[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
  }
  return as_bf16x8(make_uint4(o[0], o[1], o[2], o[3]));
}

// Eight codes as the bf16 values that they stand for.
template <int CODE>
__device__ __forceinline__ uint4 codes_to_values(uint32_t lo, uint32_t hi, float scale) {
  if constexpr (CODE == LRA_E4M3) {
    return __builtin_bit_cast(uint4, codes_to_bf16<CODE>(lo, hi, scale));
  } else {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = i < 2 ? lo : hi;
      const float a = static_cast<float>(static_cast<signed char>(w >> (16 * (i & 1)))) * scale;
      const float b = static_cast<float>(static_cast<signed char>(w >> (16 * (i & 1) + 8))) * scale;
      o[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// Integer codes have their scale in the weights: over 2^(unit - 127), at least the largest scale that the wave has met, which multiplies the
// accumulators in the end.  So the weights are within [0, 1], and rounded to bf16 as probabilities are, whatever the size of V; from 2^-127 of the unit
// down a scale counts as zero.  (With the scale itself as factor, weights of blocks below 2^-105 or so were denormal bf16 numbers of few bits.)
__device__ __forceinline__ float over_unit(int s, int unit) { return __uint_as_float(static_cast<uint32_t>(max(127 + s - unit, 0)) << 23); }
// The unit for a largest scale byte `most`: some steps above, so that blocks of about the same size seldom raise it (255 stays: no number).
__device__ __forceinline__ int unit_above(int most) { return most == 255 ? 255 : min(most + 8, 254); }

__device__ __forceinline__ uint4 masked(uint4 v, uint4 m) { return make_uint4(v.x & m.x, v.y & m.y, v.z & m.z, v.w & m.w); }

// Sequence t: its queries, and the tiles of 64 keys that they see: n_tiles in all, those from sink_tiles on `gap` further.
struct Attn8Sequence {
  int n_t, c0, c1, first_pos, lo, sinks, sink_tiles, gap, n_tiles;
};
__device__ __forceinline__ Attn8Sequence attn8_sequence(const Batch8Params& p, int t) {
  Attn8Sequence s;
  s.n_t = min(p.seq_lens[t], p.max_seq_len);
  s.c0 = t > 0 ? min(max(p.seq_query_start[t], 0), p.n_queries) : 0;
  s.c1 = t + 1 < p.n_seqs ? min(max(p.seq_query_start[t + 1], s.c0), p.n_queries) : p.n_queries;
  s.first_pos = p.causal ? s.n_t - (s.c1 - s.c0) : s.n_t - 1;
  s.lo = p.window > 0 ? max(0, s.first_pos - p.window + 1) : 0;
  s.sinks = min(p.sinks, s.lo);
  s.sink_tiles = (s.sinks + 63) / 64;
  s.gap = max(0, s.lo / 64 - s.sink_tiles);
  s.n_tiles = s.n_t <= 0 ? 0 : (s.n_t - 1) / 64 + 1 - s.gap;
  return s;
}

// Workgroup -> sequence, kv head, and which of the sequence's `shares` of the keys; false: none.  Consecutive workgroups go to
// consecutive XCDs; the kv heads of a share read the same low-rank rows, so where the shares divide by eight those go to one XCD, one
// after the other, and meet in its L2.
// Of several sequences (kShareSeqs at most) every wave forms the shares by itself: about as long as they are for head_shares of them in all, so
// that a batch of unlike lengths ends together.  With as many shares for
// every sequence 16 of 1 k to 64 k tokens (8 kv heads, 16 rows) take 234 us instead of 190, 5.6 TB/s.
__device__ __forceinline__ bool attn8_share(const Batch8Params& p, int lane, int& t, int& split, int& shares, int& h) {
  const int x = blockIdx.x, Hkv = p.n_kv_heads;
  const int eight = (x >> 3) / Hkv;
  if (p.head_shares == 0) {
    t = blockIdx.y;
    shares = p.n_splits;
    if ((p.n_splits & 7) == 0) {
      h = (x >> 3) - eight * Hkv;
      split = 8 * eight + (x & 7);
    } else {
      split = x / Hkv;
      h = x - split * Hkv;
    }
    return true;
  }
  h = (x >> 3) - eight * Hkv;
  int at = 8 * eight + (x & 7);
  constexpr int N = kShareSeqs / 64;
  int tiles[N], mine[N];
  bool queries[N];
  auto sum = [&](const int (&v)[N]) __attribute__((always_inline)) -> uint32_t {  // (fewer than 2^32: 128 times 2^24)
    uint32_t s = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) s += static_cast<uint32_t>(v[i]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += static_cast<uint32_t>(__shfl_xor(static_cast<int>(s), off, kWave));
    return __builtin_amdgcn_readfirstlane(s);
  };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Attn8Sequence s = attn8_sequence(p, min(64 * i + lane, p.n_seqs - 1));
    queries[i] = 64 * i + lane < p.n_seqs && s.c1 > s.c0;
    tiles[i] = queries[i] ? s.n_tiles : 0;
  }
  const uint32_t total = sum(tiles);
  // each sequence rounds its shares up: room for none, half or all of them
#pragma unroll 1
  for (int half = 0; half < 3; ++half) {
    const uint32_t room = max(p.head_shares - half * p.n_seqs / 2, (p.head_shares + 1) / 2);
    const uint32_t per = max((total + room - 1) / room, static_cast<uint32_t>(p.share_least));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t n = tiles[i], long_ = max(per, (n + p.n_splits - 1) / p.n_splits);
      mine[i] = queries[i] ? max(1, static_cast<int>((n + long_ - 1) / long_)) : 0;
    }
    if (sum(mine) <= static_cast<uint32_t>(p.head_shares)) break;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int upto = mine[i];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int below = __shfl_up(upto, off, kWave);
      upto += lane >= off ? below : 0;
    }
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(at < upto);
    if (beyond != 0) {
      const int k = __builtin_ctzll(beyond);
      t = 64 * i + k;
      shares = __builtin_amdgcn_readlane(mine[i], k);
      split = at - (__builtin_amdgcn_readlane(upto, k) - shares);
      return true;
    }
    at -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// The states of shares that a sequence does not have: empty, left by its first.
__device__ __forceinline__ void attn8_missing_shares(const Batch8Params& p, const Attn8Sequence& s, int n_rows, int h, int shares) {
  const int missing = p.n_splits - shares;
  for (int i = threadIdx.x; i < n_rows * missing; i += 256) {
    const int at = i / missing, tok = at / p.group;
    const int64_t row = static_cast<int64_t>(s.c0 + tok) * p.n_q_heads + h * p.group + (at - tok * p.group);
    *reinterpret_cast<float2*>(p.part_ml + (row * p.n_splits + shares + (i - at * missing)) * 2) = make_float2(-INFINITY, 0.f);
  }
}

template <int D, int RP, bool HAS_BK, int CODE>
__global__ __launch_bounds__(256, 2) void attn8_rows_kernel(Batch8Params p) {
  constexpr int NS = 4;        // waves that divide the tiles
  constexpr int KS = D / 32;   // k-steps of S^T over the head dimension
  constexpr int DB = D / 16;   // 16-row blocks of O^T
  constexpr int RB = RP / 16;  // 16-row blocks of Olr^T
  constexpr int KW = D / 64;   // 16-byte pieces of a lane's quarter of a K row
  constexpr int SLOT = ((DB + RB) * 4 + 1) * 64 * 4;  // a wave's state, lane by lane
  static_assert(RB * 64 * 8 <= 2 * SLOT);
  __shared__ __align__(16) unsigned char smem[2 * SLOT];
  __shared__ float m_s[4][16];
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hq = p.n_q_heads, Hkv = p.n_kv_heads, G = p.group, r = p.rank;
  int t, split, shares, h;
  if (!attn8_share(p, lane, t, split, shares, h)) return;
  const Attn8Sequence seq = attn8_sequence(p, t);
  const int n_t = seq.n_t, c0 = seq.c0, c1 = seq.c1, first_pos = seq.first_pos, lo = seq.lo, sinks = seq.sinks;
  const int sink_tiles = seq.sink_tiles, gap = seq.gap, n_tiles = seq.n_tiles, pos_last = n_t - 1;
  const int n_rows = min((c1 - c0) * G, 16);
  if (n_rows == 0) return;
  if (split == 0 && shares < p.n_splits) attn8_missing_shares(p, seq, n_rows, h, shares);
  // this lane's row (the last one again past the end)
  const int at_row = min(l16, n_rows - 1), tok = at_row / G;
  const int row = (c0 + tok) * Hq + h * G + (at_row - tok * G), pos = first_pos + (p.causal ? tok : 0);
  const bool live = l16 < n_rows;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / shares);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / shares);
  const int a_first = min(max(p.query_adapter[c0], 0), p.n_adapters - 1);
  const int64_t slot = static_cast<int64_t>(row) * p.n_splits + split;
  auto adapter_of_row = [&]() __attribute__((always_inline)) -> int { return p.causal ? a_first : p.query_adapter[c0 + tok]; };
  if (t0 >= t1) {
    // an empty state, all the merge kernel looks at; for a row that sees nothing at all share 0 leaves one that gives zeros
    if (wave == 0 && live) {
      const bool nothing = split == 0 && pos < 0;
      if (g == 0) {
        p.part_ml[slot * 2 + 0] = nothing ? 0.f : -INFINITY;
        p.part_ml[slot * 2 + 1] = nothing ? 1.f : 0.f;
        if (split == 0) p.part_adapter[row] = adapter_of_row();
      }
      if (nothing) {
        for (int c = g; c < D; c += 4) p.part_o[slot * D + c] = 0.f;
        for (int c = g; c < r; c += 4) p.part_lr[slot * r + c] = 0.f;
      }
    }
    return;
  }
  auto key_of = [&](int tile) __attribute__((always_inline)) -> int { return (tile < sink_tiles ? tile : tile + gap) * 64; };
  // (some query of the sequence sees it)
  auto kept = [&](int key) __attribute__((always_inline)) -> bool { return key < n_t && (key < sinks || key >= lo); };
  // whether all tokens of the tile are
  auto whole = [&](int j) __attribute__((always_inline)) -> bool { return j + 64 <= n_t && (j + 64 <= sinks || j >= lo); };

  // ---------------- a tile's requests ----------------
  const int my_block = l16 >> 2, my_token = l16 & 3;  // of the A operands of S^T: row l16
  const uint8_t* const kh = static_cast<const uint8_t*>(p.k_base) + h * p.kv_head_stride + my_token * D + g * 16;
  const uint8_t* const vh = static_cast<const uint8_t*>(p.v_base) + h * p.kv_head_stride + l16 * 16;
  const bf16_t* const lh = static_cast<const bf16_t*>(p.l) + my_token * p.l_row_stride + 4 * g;
  // id of block g of the tile; a block that nobody sees may have any: the one of the last token stands in, weighted zero
  auto look_up = [&](int j) __attribute__((always_inline)) -> int {
    const int j0 = j + 16 * g;
    const bool any = j0 < n_t && (j0 < sinks || j0 + 15 >= lo);
    return block8(p.block_table, p.max_blocks_per_seq, t, (any ? j0 : n_t - 1) >> 4);
  };
  uint4 kc[4][KW], vc[DB];
  uint2 lc[4][RB];
  int ks_raw, vs_raw;
  auto issue_k = [&](int id) __attribute__((always_inline)) {
    const uint8_t* src = kh + __shfl(id, my_block * 16, kWave) * p.kv_block_stride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int w = 0; w < KW; ++w) kc[i][w] = *reinterpret_cast<const uint4*>(src + i * 4 * D + w * 64);
    ks_raw = p.k_scale[id * p.scale_block_stride + h];
  };
  auto issue_l = [&](int id) __attribute__((always_inline)) {
    const bf16_t* src = lh + __shfl(id, my_block * 16, kWave) * static_cast<int64_t>(16) * p.l_row_stride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int b = 0; b < RB; ++b) lc[i][b] = 16 * b + 4 * g < r ? *reinterpret_cast<const uint2*>(src + 4 * i * p.l_row_stride + 16 * b) : make_uint2(0u, 0u);
  };
  auto issue_v = [&](int id) __attribute__((always_inline)) {
    const uint8_t* src = vh + id * p.kv_block_stride;
#pragma unroll
    for (int b = 0; b < DB; ++b) vc[b] = load_once(src + b * 256);
    vs_raw = p.v_scale[id * p.scale_block_stride + h];
  };
  const int first = t0 + wave;
  int id_next = 0;
  if (first < t1) {
    const int id = look_up(key_of(first));
    issue_k(id);
    issue_l(id);
    issue_v(id);
    id_next = look_up(key_of(min(first + NS, t1 - 1)));
  }

  // ---------------- prologue: Q operands, Qt = Q B_K^T ----------------
  bf16x8 qb[KS];
  {
    const bf16_t* qr = static_cast<const bf16_t*>(p.q) + static_cast<int64_t>(row) * D + g * 16;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qb[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qr + (ks >> 1) * 64 + (ks & 1) * 8));
  }
  // Qt^T, ranks by rows: register e of block b is rank 16b + 4g + e, the operand that L Qt^T takes (k = 16: four ranks a lane group).
  // Rounded to bf16, as the matrix cores take it and as lra_attn_batch has it: a score is off by 2^-8 of its adapter part at most.
  // The waves divide the queries (each with its adapter, or the chunk's one) and hand the operands round in LDS.
  s16x4v qtb[HAS_BK ? RB : 1];
  if constexpr (HAS_BK) {
    const int64_t ldb = static_cast<int64_t>(Hkv) * D;
    const int n_it = p.causal ? 1 : (n_rows - 1) / G + 1;
    uint2* const qt_s = reinterpret_cast<uint2*>(smem);
#pragma unroll 1
    for (int it = wave; it < n_it; it += NS) {
      const int a = p.causal ? a_first : min(max(p.query_adapter[c0 + it], 0), p.n_adapters - 1);
      const bf16_t* src = static_cast<const bf16_t*>(p.b_k) + static_cast<int64_t>(a) * r * ldb + h * D + g * 16;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 bk = 16 * b + l16 < r ? *reinterpret_cast<const uint4*>(src + (16 * b + l16) * ldb + (ks >> 1) * 64 + (ks & 1) * 8) : make_uint4(0u, 0u, 0u, 0u);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(bk), qb[ks], acc, 0, 0, 0);
        }
        if (p.causal || tok == it) qt_s[b * 64 + lane] = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
      }
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < RB; ++b) qtb[b] = __builtin_bit_cast(s16x4v, qt_s[b * 64 + lane]);
    __syncthreads();  // (the states go where these were)
  }
  // the identity as B operand: lane (column l16), element e <-> row 4g + e
  s16x4v eye;
#pragma unroll
  for (int e = 0; e < 4; ++e) eye[e] = 4 * g + e == l16 ? 0x3f80 : 0;

  // ---------------- main loop ----------------
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  f32x4 o_acc[DB], lr_acc[RB];
#pragma unroll
  for (int b = 0; b < DB; ++b) o_acc[b] = zero4;
#pragma unroll
  for (int b = 0; b < RB; ++b) lr_acc[b] = zero4;
  float m_run = -INFINITY, l_run = 0.f;
  int unit = 0;  // integers: what o_acc is counted in, a scale byte
  const float sc = p.scale * 1.44269504088896340736f;
  for (int tile = first; tile < t1; tile += NS) {
    const int j = key_of(tile);
    const bool more = tile + NS < t1;
    const bool all = whole(j);
    // S^T: element (i, e) of this lane is token 4i + e of block g
    // (from here to the next tile's requests the wave goes ahead of the SIMD's other one: 14 rows over 16 sequences take 141 us
    // instead of 143)
    __builtin_amdgcn_s_setprio(1);
    f32x4 s[4];
    {
      const float ks_mine = scale8(ks_raw), ks_row = __shfl(ks_mine, my_block * 16, kWave);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = zero4;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint4 c = kc[i][ks >> 1];
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<CODE>(ks & 1 ? c.z : c.x, ks & 1 ? c.w : c.y, ks_row), qb[ks], s[i], 0, 0, 0);
        }
        if constexpr (CODE == LRA_INT8) s[i] *= ks_mine;
      }
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
      for (int i = 0; i < 4; ++i) {
        const bool in = kept(j + 16 * my_block + 4 * i + my_token);
#pragma unroll
        for (int b = 0; b < RB; ++b) lc[i][b] = in ? lc[i][b] : make_uint2(0u, 0u);
      }
    }
    if constexpr (HAS_BK) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < RB; ++b) s[i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4v, lc[i][b]), qtb[b], s[i], 0, 0, 0);
    }
    if (j + 63 > first_pos) {  // some row does not see the last key
      const int last = pos - j - 16 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (4 * i + e > last) s[i][e] = -INFINITY;
    }
    if (p.window > 0 && j + p.window <= pos_last && j + 64 > p.sinks) {  // some row's window starts behind the first key
      const int from = p.sinks - j - 16 * g;
      const uint32_t hidden = static_cast<uint32_t>(max(0, pos - p.window + 1 - p.sinks));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (static_cast<uint32_t>(4 * i + e - from) < hidden) s[i][e] = -INFINITY;
    }
    // (the accumulators are rescaled only where some row's maximum grows; the probabilities, at most 1, round to bf16 for the
    // matrix cores, their sum is taken in fp32 before)
    uint32_t wl[8], wv[8];  // weights for L, and for V: with the block's scale, where that is not in V's operand
    {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[i][e]);
      mx = tile_reference(max_over_lane_groups(mx) * sc);
      if (__builtin_amdgcn_ballot_w64(mx > m_run || (CODE == LRA_INT8 && vs_raw > unit)) != 0) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
        float alpha_o = alpha;
        if constexpr (CODE == LRA_INT8) {
          int most = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) most = max(most, __builtin_amdgcn_readlane(vs_raw, 16 * i));
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
      const float vs_part = over_unit(vs_raw, unit);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(s[i][e], sc, nm));
          l_run += x[e];
        }
        wl[2 * i] = pack_bf16x2(x[0], x[1]), wl[2 * i + 1] = pack_bf16x2(x[2], x[3]);
        // (a power of two: the same rounding as without it)
        if constexpr (CODE == LRA_INT8) wv[2 * i] = pack_bf16x2(x[0] * vs_part, x[1] * vs_part), wv[2 * i + 1] = pack_bf16x2(x[2] * vs_part, x[3] * vs_part);
        else wv[2 * i] = wl[2 * i], wv[2 * i + 1] = wl[2 * i + 1];
      }
    }
    auto half = [](const uint32_t (&w)[8], int hf) __attribute__((always_inline)) { return as_bf16x8(make_uint4(w[4 * hf], w[4 * hf + 1], w[4 * hf + 2], w[4 * hf + 3])); };
    const float vs_mine = scale8(vs_raw);
    // O^T += V^T P^T: half hf of the sixteen tokens of every block
    if (!all) {  // codes of tokens that nobody sees may be no numbers: zeros
      const uint4 mask = token_masks(j + 16 * g, n_t, sinks, lo);
#pragma unroll
      for (int b = 0; b < DB; ++b) vc[b] = masked(vc[b], mask);
    }
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      o_acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<CODE>(vc[b].x, vc[b].y, vs_mine), half(wv, 0), o_acc[b], 0, 0, 0);
      o_acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<CODE>(vc[b].z, vc[b].w, vs_mine), half(wv, 1), o_acc[b], 0, 0, 0);
    }
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        // (bf16 values in fp32: their upper halves)
        auto pair = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); };
        const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4v, lc[2 * hf][b]), eye, zero4, 0, 0, 0);
        const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4v, lc[2 * hf + 1][b]), eye, zero4, 0, 0, 0);
        const bf16x8 a = as_bf16x8(make_uint4(pair(x[0], x[1]), pair(x[2], x[3]), pair(y[0], y[1]), pair(y[2], y[3])));
        lr_acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, half(wl, hf), lr_acc[b], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
    if (more) {
      issue_l(id_now);
      issue_v(id_now);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // ---------------- the waves' states: two by two through LDS, wave 0 stores ----------------
  l_run = sum_over_lane_groups(l_run);
  float m_all = m_run;
  {
    if (g == 0) m_s[wave][l16] = m_run;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NS; ++i) m_all = fmaxf(m_all, m_s[i][l16]);
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
      if (wave >= stride && wave < 2 * stride) {
        float* dst = reinterpret_cast<float*>(smem + (wave - stride) * SLOT) + lane;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) dst[(b * 4 + i) * 64] = o_acc[b][i];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) dst[((DB + b) * 4 + i) * 64] = lr_acc[b][i];
        dst[(DB + RB) * 4 * 64] = l_run;
      }
      __syncthreads();
      if (wave < stride) {
        const float* src = reinterpret_cast<const float*>(smem + wave * SLOT) + lane;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) o_acc[b][i] += src[(b * 4 + i) * 64];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) lr_acc[b][i] += src[((DB + b) * 4 + i) * 64];
        l_run += src[(DB + RB) * 4 * 64];
      }
      __syncthreads();
    }
  }
  if (wave != 0 || !live) return;
  if (g == 0) {
    const bool nothing = split == 0 && pos < 0;  // (such a row's O and O_lr are zeros)
    p.part_ml[slot * 2 + 0] = nothing ? 0.f : m_all * 0.69314718055994530942f;  // natural-log units
    p.part_ml[slot * 2 + 1] = nothing ? 1.f : l_run;
    if (split == 0) p.part_adapter[row] = adapter_of_row();
  }
#pragma unroll
  for (int b = 0; b < DB; ++b) *reinterpret_cast<f32x4*>(p.part_o + slot * D + 16 * b + 4 * g) = o_acc[b];
#pragma unroll
  for (int b = 0; b < RB; ++b)
    if (16 * b + 4 * g < r) *reinterpret_cast<f32x4*>(p.part_lr + slot * r + 16 * b + 4 * g) = lr_acc[b];  // (the rank is a multiple of 8)
}

}  // namespace lra
