// Attention of a batch over a cache of 8-bit codes: entry points and the vector-ALU kernel (contracts in lra_attn8.h).
#include <cmath>

#include "lra_attn8_plan.h"
#include "lra_codes.h"

namespace lra {

// One workgroup of four waves per (query row, share of its key tiles), 64 tokens a tile: four aligned blocks.  A quarter of a
// wave's lanes share a token's score (a quarter of its K row, of its L row each), a thread then sums one dimension of V over the
// tokens of some of the four blocks, sixteen codes a load, and one rank of L over sixteen tokens.  For fp32, ranks that are no
// multiple of 8, and as a second opinion on the MFMA kernels.  16 rows that see 260 keys take 7.5 us, the chain of a tile two to three times;
// long contexts are bound by the vector units, every row decoding its keys anew: 32 rows over 64 k tokens in fp32 167 to 173 us.
template <typename T, int D, int CODE>
__global__ __launch_bounds__(256) void attn8_vector_kernel(Batch8Params p) {
  constexpr int DQ = D / 4;             // dimensions of a K row per lane
  constexpr int VB = 4 * D / 256;       // blocks of a tile per thread (2 or 1)
  __shared__ float q_s[D], qt_s[64], s_s[64], ks_s[4], vs_s[4], o_s[256], lr_s[256];
  __shared__ __align__(16) float p_s[4][64];  // the tile's weights, of each wave for itself
  __shared__ int id_s[4];
  const int tid = threadIdx.x, lane = tid & 63;
  const int Hq = p.n_q_heads, Hkv = p.n_kv_heads, r = p.rank;
  const int row = blockIdx.x, split = blockIdx.y;
  const int tok = row / Hq, head = row - tok * Hq, h = head / p.group;
  const BatchRow b = batch_row(p, tok);
  const int64_t slot = static_cast<int64_t>(row) * p.n_splits + split;
  const int pos = b.n_keys + b.gap - 1;  // (n_keys 0: gap as it may be, nothing is seen)
  const bool nothing = b.n_keys == 0;
  const int lo = b.n_sinks + b.gap;      // first token of the window
  const int sink_tiles = (b.n_sinks + 63) / 64, gap = max(0, lo / 64 - sink_tiles);
  const int n_tiles = nothing ? 0 : pos / 64 + 1 - gap;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / p.n_splits);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / p.n_splits);
  if (split == 0 && tid == 0) p.part_adapter[row] = b.adapter;
  if (t0 >= t1) {  // an empty state, all the merge looks at; for a row that sees nothing share 0 leaves one that gives zeros
    const bool zeros = nothing && split == 0;
    if (tid == 0) {
      p.part_ml[slot * 2 + 0] = zeros ? 0.f : -INFINITY;
      p.part_ml[slot * 2 + 1] = zeros ? 1.f : 0.f;
    }
    if (zeros) {
      if (tid < D) p.part_o[slot * D + tid] = 0.f;
      if (tid < r) p.part_lr[slot * r + tid] = 0.f;
    }
    return;
  }
  if (tid < D) q_s[tid] = to_f32<T>(static_cast<const T*>(p.q)[static_cast<int64_t>(row) * D + tid]);
  __syncthreads();
  {  // Qt = q B_K^T: four lanes a rank
    const int rho = tid >> 2;
    float acc = 0.f;
    if (p.b_k != nullptr && rho < r) {
      const T* src = static_cast<const T*>(p.b_k) + (static_cast<int64_t>(b.adapter) * r + rho) * Hkv * D + static_cast<int64_t>(h) * D;
      for (int c = tid & 3; c < D; c += 4) acc = fmaf(to_f32<T>(src[c]), q_s[c], acc);
    }
    acc += __shfl_xor(acc, 1, kWave);
    acc += __shfl_xor(acc, 2, kWave);
    if ((tid & 3) == 0) qt_s[rho] = acc;
  }
  const int d_of = tid % D, part_of = tid / D;  // sums: dimension, and which of the tile's blocks
  const int rho_of = tid & 63, piece = tid >> 6;
  float m = -INFINITY, ell = 0.f, o = 0.f, olr = 0.f;
  for (int tile = t0; tile < t1; ++tile) {
    const int j = (tile < sink_tiles ? tile : tile + gap) * 64;
    __syncthreads();  // (the last tile's scores and ids have been used; Qt is there)
    if (tid < 4) {
      // a block without a visible token may have any id: the one of the query's own token stands in, weighted zero
      const int j0 = j + 16 * tid;
      const bool any = j0 <= pos && (j0 < b.n_sinks || j0 + 15 >= lo);
      const int id = block8(p.block_table, p.max_blocks_per_seq, b.t, any ? j0 >> 4 : pos >> 4);
      id_s[tid] = id;
      ks_s[tid] = scale8(p.k_scale[id * p.scale_block_stride + h]);
      vs_s[tid] = scale8(p.v_scale[id * p.scale_block_stride + h]);
    }
    __syncthreads();
    {
      const int u = tid >> 2, part = tid & 3, key = j + u;
      const int id = id_s[u >> 4];
      const bool seen = key <= pos && (key < b.n_sinks || key >= lo);
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.k_base) + id * p.kv_block_stride + h * p.kv_head_stride + (key & 15) * D + part * DQ);
      float acc = 0.f;
#pragma unroll
      for (int i = 0; i < DQ / 16; ++i) {
        const uint4 v = src[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float x[4];
          decode4<CODE>(w[c], x);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc = fmaf(x[e], q_s[part * DQ + 16 * i + 4 * c + e], acc);
        }
      }
      acc *= ks_s[u >> 4];
      if (p.b_k != nullptr) {
        const T* lrow = static_cast<const T*>(p.l) + (static_cast<int64_t>(id) * 16 + (key & 15)) * p.l_row_stride;
        for (int c = part; c < r; c += 4) acc = fmaf(to_f32<T>(lrow[c]), qt_s[c], acc);
      }
      acc += __shfl_xor(acc, 1, kWave);
      acc += __shfl_xor(acc, 2, kWave);
      if (part == 0) s_s[u] = seen ? acc * p.scale : -INFINITY;
    }
    __syncthreads();
    const float s = s_s[lane];
    // (a score below -7e8 counts as minus infinity, as a reference it would swallow the differences to it)
    const float top = wave_max(s);
    const float m_new = fmaxf(m, top < -7e8f ? -INFINITY : top);
    const float alpha = m == -INFINITY ? 0.f : expf(m - m_new);
    // (no weight where the score is minus infinity, nor where no number is above -7e8 so far; a score of NaN makes the sum one)
    const float pj = s == -INFINITY || (m_new == -INFINITY && s == s) ? 0.f : expf(s - m_new);
    m = m_new;
    ell = ell * alpha + pj;  // (of this lane's tokens)
    p_s[piece][lane] = pj;  // (by lanes' exchange instead, sixteen at a time, 200 queries of 32 heads over 2 k tokens took 733 us instead of 565)
    wave_fence();
    o *= alpha;
    olr *= alpha;
#pragma unroll
    for (int i = 0; i < VB; ++i) {
      const int blk = part_of * VB + i;
      const int id = id_s[blk];
      const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.v_base) + id * p.kv_block_stride + h * p.kv_head_stride + d_of * 16);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      float acc = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float x[4];
        decode4<CODE>(w[c], x);
        const float4 p4 = *reinterpret_cast<const float4*>(&p_s[piece][16 * blk + 4 * c]);
        const float pk[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = pk[e] == 0.f ? acc : fmaf(pk[e], x[e], acc);  // (a token that is not seen adds nothing, whatever its code)
      }
      o = fmaf(acc, vs_s[blk], o);
    }
    {
      const int id = id_s[piece];
      const T* src = static_cast<const T*>(p.l) + static_cast<int64_t>(id) * 16 * p.l_row_stride + min(rho_of, r - 1);
      T x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = src[e * p.l_row_stride];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float4 p4 = *reinterpret_cast<const float4*>(&p_s[piece][16 * piece + 4 * c]);
        const float pk[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) olr = pk[e] == 0.f ? olr : fmaf(pk[e], to_f32<T>(x[4 * c + e]), olr);
      }
    }
  }
  ell = wave_sum(ell);
  o_s[tid] = o;
  lr_s[tid] = olr;
  __syncthreads();
  if (tid < D) {
    float sum = 0.f;
    for (int i = tid; i < 256; i += D) sum += o_s[i];
    p.part_o[slot * D + tid] = sum;
  }
  if (tid < r) p.part_lr[slot * r + tid] = lr_s[tid] + lr_s[tid + 64] + lr_s[tid + 128] + lr_s[tid + 192];
  if (tid == 0) {
    p.part_ml[slot * 2 + 0] = m;
    p.part_ml[slot * 2 + 1] = ell;
  }
}

static hipError_t launch_attn8_vector(const Batch8Params& p, bool is_bf16, int rows, hipStream_t s) {
  const dim3 grid(rows, p.n_splits);
  auto launch = [&](auto t_c, auto d_c) {
    constexpr int D = decltype(d_c)::value;
    if (p.code == LRA_E4M3) hipLaunchKernelGGL((attn8_vector_kernel<decltype(t_c), D, LRA_E4M3>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attn8_vector_kernel<decltype(t_c), D, LRA_INT8>), grid, dim3(256), 0, s, p);
  };
  auto by_dim = [&](auto t_c) {
    if (p.head_dim == 128) launch(t_c, std::integral_constant<int, 128>{});
    else launch(t_c, std::integral_constant<int, 64>{});
  };
  if (is_bf16) by_dim(bf16_t{});
  else by_dim(float{});
  return hipGetLastError();
}

static Batch8Params batch8_params(const lra_shape* sh, const lra_cache8* c, const lra_adapters* ad, const lra_batch* b, const void* q) {
  Batch8Params p{};
  p.q = q;
  p.k_base = c->k;
  p.v_base = c->v;
  p.k_scale = c->k_scale;
  p.v_scale = c->v_scale;
  p.scale_block_stride = c->scale_block_stride ? c->scale_block_stride : sh->n_kv_heads;
  p.code = c->code;
  p.l = c->l;
  p.b_k = ad->b_k;
  p.b_v = ad->b_v;
  p.n_adapters = ad->n_adapters;
  p.block_table = c->block_table;
  p.seq_lens = c->seq_lens;
  p.query_adapter = b->query_adapter;
  p.seq_query_start = b->seq_query_start;
  p.kv_head_stride = c->kv_head_stride;
  p.kv_block_stride = c->kv_block_stride;
  p.l_row_stride = c->l_row_stride ? c->l_row_stride : sh->rank;
  p.n_q_heads = sh->n_q_heads;
  p.n_kv_heads = sh->n_kv_heads;
  p.group = sh->n_q_heads / sh->n_kv_heads;
  p.head_dim = sh->head_dim;
  p.rank = sh->rank;
  p.block_size = 16;
  p.max_blocks_per_seq = c->max_blocks_per_seq;
  p.num_blocks = c->num_blocks;
  p.n_seqs = c->n_seqs;
  p.max_seq_len = c->max_seq_len;
  p.n_queries = b->n_queries;
  p.max_queries_per_seq = b->max_queries_per_seq;
  p.n_new = 1;
  p.scale = sh->scale > 0.f ? sh->scale : 1.0f / std::sqrt(static_cast<float>(sh->head_dim));
  p.causal = b->causal != 0;
  // (longer ones change nothing, and sums with positions stay in 32 bits)
  p.window = b->window < c->max_seq_len ? b->window : c->max_seq_len;
  p.sinks = b->window <= 0 ? 0 : (b->sinks < c->max_seq_len ? b->sinks : c->max_seq_len);
  return p;
}

}  // namespace lra

using namespace lra;

extern "C" {

size_t lra_batch8_workspace_bytes(const lra_shape* shape, const lra_cache8* cache, const lra_batch* batch, const lra_tuning* tuning) {
  if (check_batch8(shape, cache, batch) != LRA_OK) return static_cast<size_t>(-1);
  const Attn8Plan pl = plan_attn8(shape, cache, batch, resolve_tuning(tuning));
  return pl.launchable ? pl.bytes : static_cast<size_t>(-1);
}

lra_status lra_attn_batch8(const lra_shape* shape, const lra_cache8* cache, const lra_adapters* adapters, const lra_batch* batch,
                           const void* q, void* out, void* workspace, size_t workspace_bytes, const lra_tuning* tuning, void* stream) {
  const lra_status st = check_batch8(shape, cache, batch);
  if (st != LRA_OK) return st;
  if (!adapters || !q || !out) return LRA_ERR_NULL;
  if (adapters->n_adapters < 1) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(adapters->b_k) |
       reinterpret_cast<uintptr_t>(adapters->b_v)) & 15)
    return LRA_ERR_SHAPE;
  if (shape->key_rope_theta > 0.f && adapters->b_k) return LRA_ERR_UNSUPPORTED;
  const Attn8Plan pl = plan_attn8(shape, cache, batch, resolve_tuning(tuning));
  if (!pl.launchable) return LRA_ERR_UNSUPPORTED;
  if (pl.bytes > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < pl.bytes)) return LRA_ERR_WORKSPACE;
  Batch8Params p = batch8_params(shape, cache, adapters, batch, q);
  p.out = out;
  p.n_splits = pl.n_splits;
  p.head_shares = pl.head_shares;
  p.share_least = pl.share_least;
  if (pl.states) {
    char* ws = static_cast<char*>(workspace);
    p.part_ml = reinterpret_cast<float*>(ws + pl.off_ml);
    p.part_o = reinterpret_cast<float*>(ws + pl.off_o);
    p.part_lr = reinterpret_cast<float*>(ws + pl.off_lr);
    p.part_adapter = reinterpret_cast<int32_t*>(ws + pl.off_adapter);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = shape->dtype == LRA_BF16;
  if (pl.few_rows) {
    if ((p.code == LRA_E4M3 ? launch_attn8_rows_e4m3 : launch_attn8_rows_int8)(p, pl.row_tiles, s) != hipSuccess) return LRA_ERR_HIP;
  } else if (pl.tiles) {
    p.row_mul = (65535 + p.group) / p.group;
    p.tile_places = pl.tile_places;
    p.longest_first = pl.longest_first;
    if ((p.code == LRA_E4M3 ? launch_attn8_tiles_e4m3 : launch_attn8_tiles_int8)(p, s) != hipSuccess) return LRA_ERR_HIP;
  } else if (launch_attn8_vector(p, bf16, pl.rows, s) != hipSuccess) {
    return LRA_ERR_HIP;
  }
  if (pl.states && launch_merge(p, bf16, pl.rows, s) != hipSuccess) return LRA_ERR_HIP;
  return LRA_OK;
}

}  // extern "C"
