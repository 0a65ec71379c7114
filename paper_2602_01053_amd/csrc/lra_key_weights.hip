// Attention weight per cached token: entry points and vector-ALU kernels of lra_key_weights (fp32, ranks that are no multiple of
// 8, one low-rank cache per adapter); bf16 runs on lra_key_weights_mfma.hip.
//
// Two passes over the keys, since a weight needs its row's maximum and sum first:
//   Qt    = Q B_K^T of every query row                                        (once, to the workspace)
//   lse   = log2 sum_j exp2(s_j), s = scale log2(e) (Q K_base^T + Qt L^T)     per row
//   w[j] += sum over rows exp2(s_j - lse)                                     per key, rows added up in a fixed order
#include "lra_attn.h"
#include "lra_batch.h"
#include "lra_batch_plan.h"
#include "lra_decode_util.h"
#include "lra_key_weights.h"

#include <cmath>

namespace lra {

constexpr float kLog2e = 1.44269504088896340736f;

// Row idx of the batch: query idx / Hq, q head idx % Hq.

// A row's Q . K of token j, the K row in 16-byte pieces, sixteen requested before the first is used
template <typename T, int D>
__device__ __forceinline__ float dot_key(const WeightsParams& p, int t, int j, int h, const float* q) {
  constexpr int E = 16 / static_cast<int>(sizeof(T)), N = D / E, U = N < 16 ? N : 16;
  const u32x4* k = reinterpret_cast<const u32x4*>(static_cast<const T*>(p.k_base) + kv_offset(p, t, j, h));
  float acc = 0.f;
#pragma unroll
  for (int c0 = 0; c0 < N; c0 += U) {
    u32x4 v[U];
#pragma unroll
    for (int c = 0; c < U; ++c) v[c] = k[c0 + c];
#pragma unroll
    for (int c = 0; c < U; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float x;
        if constexpr (sizeof(T) == 4) x = __uint_as_float(v[c][e]);
        else x = __uint_as_float((e & 1) ? (v[c][e >> 1] & 0xffff0000u) : (v[c][e >> 1] << 16));
        acc = fmaf(x, q[(c0 + c) * E + e], acc);
      }
  }
  return acc;
}

// scale log2(e) times the score of a row (q and Qt in LDS) and a key; the low-rank row eight elements at a time, past its end the
// last one again against zeros of Qt
template <typename T, int D>
__device__ __forceinline__ float score(const WeightsParams& p, int t, int j, int h, int a, const float* q, const float* qt) {
  float low = 0.f;
  if (p.b_k != nullptr) {
    const T* l = static_cast<const T*>(p.l) + l_offset(p, t, j, a);
    for (int r0 = 0; r0 < p.rank; r0 += 8) {
      T v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = l[min(r0 + e, p.rank - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e) low = fmaf(to_f32<T>(v[e]), qt[r0 + e], low);
    }
  }
  return (dot_key<T, D>(p, t, j, h, q) + low) * (p.scale * kLog2e);
}

// One workgroup per row and key share; a lane takes every 256th key.  Qt of the row is formed here, four lanes to a rank, and left
// for the sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void weights_stats_kernel(WeightsParams p, int64_t rows) {
  __shared__ float q[D], qt[64], m_s[4], l_s[4];
  const int tid = threadIdx.x, split = blockIdx.y;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int tok = static_cast<int>(row / p.n_q_heads), h = static_cast<int>(row % p.n_q_heads) / p.group;
    const BatchRow b = batch_row(p, tok);
    __syncthreads();
    if (tid < D) q[tid] = to_f32<T>(static_cast<const T*>(p.q)[row * D + tid]);
    __syncthreads();
    {
      const int rho = tid >> 2, part = tid & 3;
      float acc = 0.f;
      if (p.b_k != nullptr && rho < p.rank) {
        const T* bk = static_cast<const T*>(p.b_k) + ((static_cast<int64_t>(b.adapter) * p.rank + rho) * p.n_kv_heads + h) * D;
#pragma unroll 16
        for (int c = 0; c < D / 4; ++c) acc = fmaf(q[4 * c + part], to_f32<T>(bk[4 * c + part]), acc);
      }
      acc += __shfl_xor(acc, 1, kWave);
      acc += __shfl_xor(acc, 2, kWave);
      if (part == 0) {
        qt[rho] = acc;
        if (p.b_k != nullptr && rho < p.rank && split == 0) p.qt[row * p.rank + rho] = acc;
      }
    }
    __syncthreads();
    float m = -INFINITY, l = 0.f;
    const int k1 = static_cast<int>(static_cast<int64_t>(b.n_keys) * (split + 1) / p.n_splits);
    for (int k = static_cast<int>(static_cast<int64_t>(b.n_keys) * split / p.n_splits) + tid; k < k1; k += 256) {
      const float s = score<T, D>(p, b.t, k < b.n_sinks ? k : k + b.gap, h, b.adapter, q, qt);
      if (s == -INFINITY) continue;
      const float m_new = fmaxf(m, s);
      l = l * exp2f(m - m_new) + exp2f(s - m_new);
      m = m_new;
    }
    const float top_w = wave_max(m);
    const float sum_w = wave_sum(m == -INFINITY ? l : l * exp2f(m - top_w));
    const int wave = tid >> 6;
    if ((tid & 63) == 0) {
      m_s[wave] = top_w;
      l_s[wave] = sum_w;
    }
    __syncthreads();
    if (tid == 0) {
      const float top = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3]));
      float sum = 0.f;
      for (int w = 0; w < 4; ++w) sum += m_s[w] == -INFINITY ? l_s[w] : l_s[w] * exp2f(m_s[w] - top);
      reinterpret_cast<float2*>(p.stats)[row * p.n_splits + split] = make_float2(top, sum);
    }
  }
}

// One workgroup per (64 keys, sequence); a wave takes every sixteenth row of the sequence, a lane one key.
template <typename T, int D>
__global__ __launch_bounds__(1024) void weights_sum_kernel(WeightsParams p) {
  __shared__ float q[16][D], qt[16][64], sum_s[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.y;
  const int j = blockIdx.x * 64 + lane;
  const int n_t = min(p.seq_lens[t], p.max_seq_len);
  if (static_cast<int>(blockIdx.x) * 64 >= n_t) return;
  const int c0 = t > 0 ? p.seq_query_start[t] : 0, c1 = t + 1 < p.n_seqs ? p.seq_query_start[t + 1] : p.n_queries;
  float sum = 0.f;
  for (int64_t row = static_cast<int64_t>(c0) * p.n_q_heads + wave; row < static_cast<int64_t>(c1) * p.n_q_heads; row += 16) {
    const int tok = static_cast<int>(row / p.n_q_heads), h = static_cast<int>(row % p.n_q_heads) / p.group;
    // the shares' statistics joined, a lane each (32 at most)
    const float2 ml = lane < p.n_splits ? reinterpret_cast<const float2*>(p.stats)[row * p.n_splits + lane] : make_float2(-INFINITY, 0.f);
    const float top = wave_max(ml.x);
    const float all = wave_sum(ml.x == -INFINITY ? ml.y : ml.y * exp2f(ml.x - top));  // (a share's NaN is the row's)
    if (all == 0.f) continue;  // the row sees nothing
    const float lse = top + log2f(all);
    for (int c = lane; c < D; c += 64) q[wave][c] = to_f32<T>(static_cast<const T*>(p.q)[row * D + c]);
    qt[wave][lane] = p.b_k != nullptr && lane < p.rank ? p.qt[row * p.rank + lane] : 0.f;
    lds_fence();
    const int pos = p.causal ? n_t - (c1 - tok) : n_t - 1;
    const int a = min(max(p.query_adapter[p.causal ? c0 : tok], 0), p.n_adapters - 1);
    if (j < n_t && batch_sees(p, pos, j)) sum += exp2f(score<T, D>(p, t, j, h, a, q[wave], qt[wave]) - lse);
    lds_fence();
  }
  sum_s[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && j < n_t) {
    float* w = p.weights + t * p.weights_stride + j;
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) all += sum_s[i][lane];
    *w = p.decay == 0.f ? all : fmaf(p.decay, *w, all);
  }
}

template <typename T, int D>
static hipError_t launch_weights(const WeightsParams& p, int rows, hipStream_t s) {
  hipLaunchKernelGGL((weights_stats_kernel<T, D>), dim3(static_cast<unsigned>(rows < 65536 ? rows : 65536), p.n_splits), dim3(256), 0, s, p, static_cast<int64_t>(rows));
  hipLaunchKernelGGL((weights_sum_kernel<T, D>), dim3((p.max_seq_len + 63) / 64, p.n_seqs), dim3(1024), 0, s, p);
  return hipGetLastError();
}

template <typename T>
static hipError_t launch_weights_t(const WeightsParams& p, int rows, hipStream_t s) {
  return p.head_dim == 128 ? launch_weights<T, 128>(p, rows, s) : launch_weights<T, 64>(p, rows, s);
}

}  // namespace lra

using namespace lra;

extern "C" {

static lra_status check_key_weights(const lra_shape* shape, const lra_cache* cache, const lra_batch* batch) {
  const lra_status st = check_batch(shape, cache, batch);
  if (st != LRA_OK) return st;
  if (cache->n_seqs > 65535) return LRA_ERR_UNSUPPORTED;  // (sequences in a grid's y)
  return LRA_OK;
}

size_t lra_key_weights_workspace_bytes(const lra_shape* shape, const lra_cache* cache, const lra_batch* batch, const lra_tuning* tuning) {
  if (check_key_weights(shape, cache, batch) != LRA_OK) return static_cast<size_t>(-1);
  return plan_key_weights(shape, cache, batch, resolve_tuning(tuning)).bytes;
}

lra_status lra_key_weights(const lra_shape* shape, const lra_cache* cache, const lra_adapters* adapters, const lra_batch* batch,
                           const void* q, float decay, float* weights, int64_t weights_stride, void* workspace,
                           size_t workspace_bytes, const lra_tuning* tuning, void* stream) {
  const lra_status st = check_key_weights(shape, cache, batch);
  if (st != LRA_OK) return st;
  if (!adapters || !q || !weights) return LRA_ERR_NULL;
  if (adapters->n_adapters < 1 || weights_stride < cache->max_seq_len || !std::isfinite(decay)) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(adapters->b_k)) & 15) return LRA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(weights) & 3) return LRA_ERR_SHAPE;
  if (shape->key_rope_theta > 0.f && adapters->b_k) return LRA_ERR_UNSUPPORTED;
  const WeightsPlan pl = plan_key_weights(shape, cache, batch, resolve_tuning(tuning));
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < pl.bytes) return LRA_ERR_WORKSPACE;
  WeightsParams p{};
  static_cast<BatchParams&>(p) = batch_params(shape, cache, adapters, batch, q);
  char* ws = static_cast<char*>(workspace);
  p.qt = reinterpret_cast<float*>(ws + pl.off_qt);
  p.lse = reinterpret_cast<float*>(ws + pl.off_lse);
  p.stats = reinterpret_cast<float*>(ws + pl.off_stats);
  p.n_splits = pl.n_splits;
  p.sum_groups = pl.sum_groups;
  p.group_sums = reinterpret_cast<float*>(ws + pl.off_sums);
  p.rows_per_head = batch->n_queries * p.group;
  p.row_mul = (65535 + p.group) / p.group;
  p.tile_places = pl.tile_places;
  p.weights = weights;
  p.weights_stride = weights_stride;
  p.decay = decay;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t err = pl.mfma ? launch_key_weights_mfma(p, s)
                         : shape->dtype == LRA_BF16 ? launch_weights_t<bf16_t>(p, pl.rows, s)
                                                    : launch_weights_t<float>(p, pl.rows, s);
  return err == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
