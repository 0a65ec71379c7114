// Attention weight per cached token on the matrix cores (bf16 caches with one L): lra_key_weights of the header.
//
//   Qt    = Q B_K^T, as two bf16 terms (16 bits of mantissa: the second is what the first left over)
//   stats: per query row and key share  m = max s, l = sum exp2(s - m),  s = scale log2(e) (K_base Q^T + L Qt^T)
//   lse   = m + log2 l over the shares
//   sums:  w[j] = decay w[j] + sum over rows exp2(s_j - lse)
//
// Scores are products of bf16 in fp32, so the weights come out as exactly as fp32 sums of them allow; Qt rounded to one
// bf16 term alone would put 1e-3 into each.  Both passes hold 64 keys of a kv head in registers as the A operand of
// v_mfma_f32_32x32x16_bf16 and take the query rows past them 32 at a time: what differs is who owns what.  In the
// statistics a workgroup owns a key share of one kv head and its waves take its 64-key tiles in turn, the running m and l of
// a row kept per lane in LDS; in the sums it owns 64 keys of all kv heads and its waves divide the (head, 32 rows) blocks, so
// that the sum over heads and rows stays in the workgroup, is added up in one fixed order, and needs no atomics.
// K rows go from memory to registers (two 16-byte pieces of a row per lane pair and load; a row's eight loads use its lines
// whole), since no two waves of a workgroup share them.
#include "lra_decode_util.h"
#include "lra_key_weights.h"
#include "lra_prefill_util.h"

namespace lra {

// One workgroup per (query, kv head); a group of D / 8 lanes per rank.
template <int D, int RP>
__global__ __launch_bounds__(256) void weights_qt_mfma_kernel(WeightsParams p) {
  constexpr int LPR = D / 8;
  const int tok = blockIdx.x, h = blockIdx.y, r = p.rank, G = p.group;
  const int grp = threadIdx.x / LPR, c = threadIdx.x % LPR;
  int a = p.query_adapter[tok];
  if (p.causal) {
    const int t = p.n_seqs > 1 ? sequence_of_query(p, tok) : 0;
    a = p.query_adapter[t > 0 ? p.seq_query_start[t] : 0];
  }
  a = min(max(a, 0), p.n_adapters - 1);
  const bf16_t* q = static_cast<const bf16_t*>(p.q) + (static_cast<int64_t>(tok) * p.n_q_heads + h * G) * D + c * 8;
  const bf16_t* b = static_cast<const bf16_t*>(p.b_k) + (static_cast<int64_t>(a) * r * p.n_kv_heads + h) * D + c * 8;
  bf16_t* qt = reinterpret_cast<bf16_t*>(p.qt) + (static_cast<int64_t>(h) * p.rows_per_head + static_cast<int64_t>(tok) * G) * 2 * RP;
  for (int rho = grp; rho < RP; rho += 256 / LPR) {
    u32x4 bp = {0u, 0u, 0u, 0u};
    if (rho < r) bp = *reinterpret_cast<const u32x4*>(b + static_cast<int64_t>(rho) * p.n_kv_heads * D);
    for (int g = 0; g < G; ++g) {
      const u32x4 qp = *reinterpret_cast<const u32x4*>(q + g * D);
      float acc = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc = fmaf(__uint_as_float(bp[e] << 16), __uint_as_float(qp[e] << 16), acc);
        acc = fmaf(__uint_as_float(bp[e] & 0xffff0000u), __uint_as_float(qp[e] & 0xffff0000u), acc);
      }
#pragma unroll
      for (int off = LPR / 2; off > 0; off >>= 1) acc += __shfl_xor(acc, off, kWave);
      if (c == 0) {
        const bf16_t hi = f32_to_bf16(acc);
        const float rest = acc - bf16_to_f32(hi);
        qt[g * 2 * RP + rho] = hi;
        qt[g * 2 * RP + RP + rho] = f32_to_bf16(__builtin_isfinite(rest) ? rest : 0.f);
      }
    }
  }
}

// What the queries of a sequence see: [0, sinks) and [lo, n_t).
struct WeightsSeq {
  int t, c0, c1, n_t, sinks, lo;
};
__device__ __forceinline__ WeightsSeq weights_seq(const WeightsParams& p, int t) {
  WeightsSeq s;
  s.t = t;
  s.c0 = t > 0 ? min(max(PF_CONST_I32(p.seq_query_start)[t], 0), p.n_queries) : 0;
  s.c1 = t + 1 < p.n_seqs ? min(max(PF_CONST_I32(p.seq_query_start)[t + 1], s.c0), p.n_queries) : p.n_queries;
  s.n_t = min(PF_CONST_I32(p.seq_lens)[t], p.max_seq_len);
  const int first = p.causal ? s.n_t - (s.c1 - s.c0) : s.n_t - 1;
  s.lo = p.window > 0 ? max(0, first - p.window + 1) : 0;
  s.sinks = min(p.sinks, s.lo);
  return s;
}

// 64 keys of a kv head as A operands: lane (key 32 kt + l32, half g2), element e of k-step ks <-> feature 16 ks + 8 g2 + e.
template <int D, int RP, bool HAS_BK, bool PAGED>
struct KeyOperands {
  static constexpr int KS = D / 16, RKS = HAS_BK ? RP / 16 : 1;
  pf_bf16x8 k[2][KS], l[2][RKS];
  // tokens that no query sees, or past the end: the last token in their place (masked later)
  __device__ __forceinline__ void load(const WeightsParams& p, const WeightsSeq& s, int j, int h, int l32, int g2) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      int key = j + 32 * kt + l32;
      if (!(key < s.n_t && (key < s.sinks || key >= s.lo))) key = s.n_t - 1;
      int64_t row = key, off;
      if constexpr (PAGED) {
        const int blk = p.block_table[static_cast<int64_t>(s.t) * p.max_blocks_per_seq + (key >> 4)];
        off = blk * p.kv_block_stride + (key & 15) * p.kv_token_stride;
        row = static_cast<int64_t>(blk) * 16 + (key & 15);
      } else {
        off = key * p.kv_token_stride;
      }
      const bf16_t* kr = static_cast<const bf16_t*>(p.k_base) + off + static_cast<int64_t>(h) * p.kv_head_stride + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[kt][ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(kr + ks * 16));
      if constexpr (HAS_BK) {
        const bf16_t* lr = static_cast<const bf16_t*>(p.l) + row * p.l_row_stride;
#pragma unroll
        for (int ks = 0; ks < RKS; ++ks)  // (the rank is a multiple of 8; past it the last eight again, against zeros of Qt)
          l[kt][ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(lr + min(16 * ks + 8 * g2, p.rank - 8)));
      }
    }
  }
};

// 32 query rows as B operands: lane (row l32 of the block, half g2)
template <int D, int RP, bool HAS_BK>
struct RowOperands {
  static constexpr int KS = D / 16, RKS = HAS_BK ? RP / 16 : 1;
  pf_bf16x8 q[KS], hi[RKS], lo[RKS];
  __device__ __forceinline__ void load(const WeightsParams& p, int h, int row, int g2) {
    const int tok = row / p.group, g = row - tok * p.group;
    const bf16_t* qr = static_cast<const bf16_t*>(p.q) + (static_cast<int64_t>(tok) * p.n_q_heads + h * p.group + g) * D + g2 * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qr + ks * 16));
    if constexpr (HAS_BK) {
      const bf16_t* qt = reinterpret_cast<const bf16_t*>(p.qt) + (static_cast<int64_t>(h) * p.rows_per_head + row) * 2 * RP + g2 * 8;
#pragma unroll
      for (int ks = 0; ks < RKS; ++ks) {
        hi[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qt + ks * 16));
        lo[ks] = __builtin_bit_cast(pf_bf16x8, *reinterpret_cast<const pf_u32x4*>(qt + RP + ks * 16));
      }
    }
  }
};

// Scores of 64 keys and 32 rows: s[kt][i] is key 32 kt + 8 (i / 4) + 4 g2 + i % 4 of row l32, minus infinity where it is not seen.
template <int D, int RP, bool HAS_BK, bool PAGED>
__device__ __forceinline__ void block_scores(const WeightsParams& p, const WeightsSeq& sq, const KeyOperands<D, RP, HAS_BK, PAGED>& key,
                                             const RowOperands<D, RP, HAS_BK>& row, int j, int pos, int pos_first, int pos_last, int g2,
                                             pf_f32x16 (&s)[2]) {
  constexpr int KS = D / 16, RKS = RP / 16;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
  if constexpr (HAS_BK) {
#pragma unroll
    for (int ks = 0; ks < RKS; ++ks) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key.l[kt][ks], row.lo[ks], s[kt], 0, 0, 0);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key.l[kt][ks], row.hi[ks], s[kt], 0, 0, 0);
    }
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key.k[kt][ks], row.q[ks], s[kt], 0, 0, 0);
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

template <int D, int RP, bool HAS_BK, bool PAGED>
__global__ __launch_bounds__(256, 2) void weights_stats_mfma_kernel(WeightsParams p) {
  __shared__ float2 ml_s[4][kWeightRows / 32][64];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x / p.n_kv_heads, h = blockIdx.x - split * p.n_kv_heads;
  const WeightsSeq sq = weights_seq(p, blockIdx.y);
  const int G = p.group;
  const int row_first = sq.c0 * G + static_cast<int>(blockIdx.z) * kWeightRows;
  const int row_end = min(sq.c1 * G, row_first + kWeightRows);
  if (row_first >= row_end) return;
  const int blocks = (row_end - row_first + 31) / 32;
  // 64-key tiles of what the sequence's queries see (as in batch_tiles_body), this share's, and of those every fourth
  const int sink_tiles = (sq.sinks + 63) / 64, gap = max(0, sq.lo / 64 - sink_tiles);
  const int n_tiles = sq.n_t <= 0 ? 0 : (sq.n_t - 1) / 64 + 1 - gap;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / p.n_splits);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / p.n_splits);
  for (int b = 0; b < blocks; ++b) ml_s[wave][b][lane] = make_float2(-INFINITY, 0.f);
  const float sc = p.scale * 1.44269504088896340736f;
  auto pos_of = [&](int row) __attribute__((always_inline)) -> int { return p.causal ? sq.n_t - (sq.c1 - row / G) : sq.n_t - 1; };
  for (int tile = t0 + wave; tile < t1; tile += 4) {
    const int j = (tile < sink_tiles ? tile : tile + gap) * 64;
    KeyOperands<D, RP, HAS_BK, PAGED> key;
    key.load(p, sq, j, h, l32, g2);
    for (int b = 0; b < blocks; ++b) {
      const int r0 = row_first + 32 * b, r1 = min(r0 + 31, row_end - 1);
      const int pos_first = pos_of(r0), pos_last = pos_of(r1);
      if (j > pos_last || (p.window > 0 && j + 63 + p.window <= pos_first && j >= p.sinks)) continue;  // nothing of the tile is seen
      const int row = min(r0 + l32, r1);
      RowOperands<D, RP, HAS_BK> rows;
      rows.load(p, h, row, g2);
      pf_f32x16 s[2];
      block_scores<D, RP, HAS_BK, PAGED>(p, sq, key, rows, j, pos_of(row), pos_first, pos_last, g2, s);
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
      float2 ml = ml_s[wave][b][lane];
      const float m = fmaxf(ml.x, mx * sc);
      const float nm = m == -INFINITY ? 0.f : -m;
      float sum = ml.y * __builtin_amdgcn_exp2f(ml.x + nm);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, nm));
      ml_s[wave][b][lane] = make_float2(m, sum);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < row_end - row_first; i += 256) {
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float2 x = ml_s[w][i >> 5][(i & 31) + 32 * g];
        const float m_new = fmaxf(m, x.x);
        const float nm = m_new == -INFINITY ? 0.f : -m_new;
        l = l * __builtin_amdgcn_exp2f(m + nm) + x.y * __builtin_amdgcn_exp2f(x.x + nm);
        m = m_new;
      }
    float* out = p.stats + ((static_cast<int64_t>(h) * p.n_splits + split) * p.rows_per_head + row_first + i) * 2;
    *reinterpret_cast<float2*>(out) = make_float2(m, l);
  }
}

__global__ __launch_bounds__(256) void weights_lse_kernel(WeightsParams p) {
  const int row = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y;
  if (row >= p.rows_per_head) return;
  const float2* ml = reinterpret_cast<const float2*>(p.stats) + static_cast<int64_t>(h) * p.n_splits * p.rows_per_head + row;
  float m = -INFINITY;
  for (int s = 0; s < p.n_splits; ++s) m = fmaxf(m, ml[static_cast<int64_t>(s) * p.rows_per_head].x);
  const float nm = m == -INFINITY ? 0.f : -m;
  float l = 0.f;
  for (int s = 0; s < p.n_splits; ++s) {
    const float2 x = ml[static_cast<int64_t>(s) * p.rows_per_head];
    l = fmaf(x.y, __builtin_amdgcn_exp2f(x.x + nm), l);
  }
  p.lse[static_cast<int64_t>(h) * p.rows_per_head + row] = l == 0.f ? INFINITY : m + log2f(l);
}

template <int D, int RP, bool HAS_BK, bool PAGED>
__global__ __launch_bounds__(256, 2) void weights_sum_mfma_kernel(WeightsParams p) {
  __shared__ float sum_s[4][64];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x * 64;
  const WeightsSeq sq = weights_seq(p, blockIdx.y);
  if (j >= sq.n_t) return;
  const int G = p.group;
  const float sc = p.scale * 1.44269504088896340736f;
  auto pos_of = [&](int row) __attribute__((always_inline)) -> int { return p.causal ? sq.n_t - (sq.c1 - row / G) : sq.n_t - 1; };
  pf_f32x16 acc[2];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[kt][i] = 0.f;
  const int rows = (sq.c1 - sq.c0) * G, blocks = (rows + 31) / 32;
  if (rows > 0 && (j < sq.sinks || j + 63 >= sq.lo)) {
    const int items = p.n_kv_heads * blocks;  // (at most 2^30 rows / 32)
    int left = static_cast<int>(static_cast<int64_t>(items) * (wave + 1) / 4);
    int h = static_cast<int>(static_cast<int64_t>(items) * wave / 4);
    left -= h;
    int b = h;
    h /= blocks;
    b -= h * blocks;
    for (; left > 0; ++h) {
      KeyOperands<D, RP, HAS_BK, PAGED> key;
      key.load(p, sq, j, h, l32, g2);
      for (; b < blocks && left > 0; ++b, --left) {
        const int r0 = sq.c0 * G + 32 * b, r1 = min(r0 + 31, sq.c1 * G - 1);
        const int pos_first = pos_of(r0), pos_last = pos_of(r1);
        if (j > pos_last || (p.window > 0 && j + 63 + p.window <= pos_first && j >= p.sinks)) continue;
        const int row = min(r0 + l32, r1);
        RowOperands<D, RP, HAS_BK> ro;
        ro.load(p, h, row, g2);
        const float lse = p.lse[static_cast<int64_t>(h) * p.rows_per_head + row];
        pf_f32x16 s[2];
        block_scores<D, RP, HAS_BK, PAGED>(p, sq, key, ro, j, pos_of(row), pos_first, pos_last, g2, s);
        const float nl = r0 + l32 <= r1 ? -lse : -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[kt][i] += __builtin_amdgcn_exp2f(fmaf(s[kt][i], sc, nl));
      }
      b = 0;
    }
  }
  // over the 32 lanes of a half (its rows), then the waves
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = acc[kt][i];
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
      if (l32 == 0) sum_s[wave][32 * kt + 8 * (i >> 2) + 4 * g2 + (i & 3)] = v;
    }
  __syncthreads();
  if (wave == 0 && j + lane < sq.n_t) {
    float* w = p.weights + sq.t * p.weights_stride + j + lane;
    const float all = (sum_s[0][lane] + sum_s[1][lane]) + (sum_s[2][lane] + sum_s[3][lane]);
    *w = p.decay == 0.f ? all : fmaf(p.decay, *w, all);
  }
}

template <int D, int RP, bool HAS_BK, bool PAGED>
static void launch_passes(const WeightsParams& p, hipStream_t s) {
  if constexpr (HAS_BK) hipLaunchKernelGGL((weights_qt_mfma_kernel<D, RP>), dim3(p.n_queries, p.n_kv_heads), dim3(256), 0, s, p);
  const int row_groups = static_cast<int>((static_cast<int64_t>(p.max_queries_per_seq) * p.group + kWeightRows - 1) / kWeightRows);
  hipLaunchKernelGGL((weights_stats_mfma_kernel<D, RP, HAS_BK, PAGED>), dim3(p.n_kv_heads * p.n_splits, p.n_seqs, row_groups), dim3(256), 0, s, p);
  hipLaunchKernelGGL(weights_lse_kernel, dim3((p.rows_per_head + 255) / 256, p.n_kv_heads), dim3(256), 0, s, p);
  hipLaunchKernelGGL((weights_sum_mfma_kernel<D, RP, HAS_BK, PAGED>), dim3((p.max_seq_len + 63) / 64, p.n_seqs), dim3(256), 0, s, p);
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
