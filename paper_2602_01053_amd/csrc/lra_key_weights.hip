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
template <typename T>
__global__ __launch_bounds__(256) void weights_qt_kernel(WeightsParams p, int64_t n) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;  // (row, rank)
  if (at >= n) return;
  const int64_t row = at / p.rank;
  const int rho = static_cast<int>(at - row * p.rank), d = p.head_dim;
  const int tok = static_cast<int>(row / p.n_q_heads), h = static_cast<int>(row % p.n_q_heads) / p.group;
  const int a = batch_row(p, tok).adapter;
  const T* q = static_cast<const T*>(p.q) + row * d;
  const T* b = static_cast<const T*>(p.b_k) + ((static_cast<int64_t>(a) * p.rank + rho) * p.n_kv_heads + h) * d;
  float acc = 0.f;
  for (int c = 0; c < d; ++c) acc = fmaf(to_f32<T>(q[c]), to_f32<T>(b[c]), acc);
  p.qt[at] = acc;
}

// scale log2(e) times the score of a row (q in LDS, Qt) and a key
template <typename T>
__device__ __forceinline__ float score(const WeightsParams& p, int t, int j, int h, int a, const float* q, const float* qt) {
  const T* k = static_cast<const T*>(p.k_base) + kv_offset(p, t, j, h);
  constexpr int PER = 16 / static_cast<int>(sizeof(T));
  float acc = 0.f;
  for (int c = 0; c < p.head_dim; c += PER) {
    const uint4 piece = *reinterpret_cast<const uint4*>(k + c);
    const uint32_t w[4] = {piece.x, piece.y, piece.z, piece.w};
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      float x;
      if constexpr (sizeof(T) == 4) x = __uint_as_float(w[e]);
      else x = __uint_as_float((e & 1) ? (w[e >> 1] & 0xffff0000u) : (w[e >> 1] << 16));
      acc = fmaf(x, q[c + e], acc);
    }
  }
  if (p.b_k != nullptr) {
    const T* l = static_cast<const T*>(p.l) + l_offset(p, t, j, a);
    for (int rho = 0; rho < p.rank; ++rho) acc = fmaf(to_f32<T>(l[rho]), qt[rho], acc);
  }
  return acc * (p.scale * kLog2e);
}

template <typename T>
__device__ __forceinline__ void stage_row(const WeightsParams& p, int64_t row, float* q, float* qt, int first, int step) {
  for (int c = first; c < p.head_dim; c += step) q[c] = to_f32<T>(static_cast<const T*>(p.q)[row * p.head_dim + c]);
  if (p.b_k != nullptr)
    for (int c = first; c < p.rank; c += step) qt[c] = p.qt[row * p.rank + c];
}

// One workgroup per row; a lane takes every 256th key.
template <typename T>
__global__ __launch_bounds__(256) void weights_stats_kernel(WeightsParams p, int64_t rows) {
  __shared__ float q[128], qt[64], m_s[4], l_s[4];
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int tok = static_cast<int>(row / p.n_q_heads), h = static_cast<int>(row % p.n_q_heads) / p.group;
    const BatchRow b = batch_row(p, tok);
    __syncthreads();
    stage_row<T>(p, row, q, qt, threadIdx.x, 256);
    __syncthreads();
    float m = -INFINITY, l = 0.f;
    for (int k = threadIdx.x; k < b.n_keys; k += 256) {
      const float s = score<T>(p, b.t, k < b.n_sinks ? k : k + b.gap, h, b.adapter, q, qt);
      if (s == -INFINITY) continue;
      const float m_new = fmaxf(m, s);
      l = l * exp2f(m - m_new) + exp2f(s - m_new);
      m = m_new;
    }
    const float top_w = wave_max(m);
    const float sum_w = wave_sum(m == -INFINITY ? l : l * exp2f(m - top_w));
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      m_s[wave] = top_w;
      l_s[wave] = sum_w;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      const float top = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3]));
      float sum = 0.f;
      for (int w = 0; w < 4; ++w) sum += m_s[w] == -INFINITY ? l_s[w] : l_s[w] * exp2f(m_s[w] - top);
      p.lse[row] = sum == 0.f ? -INFINITY : top + log2f(sum);
    }
  }
}

// One workgroup per (64 keys, sequence); a wave takes every fourth row of the sequence, a lane one key.
template <typename T>
__global__ __launch_bounds__(256) void weights_sum_kernel(WeightsParams p) {
  __shared__ float q[4][128], qt[4][64], sum_s[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.y;
  const int j = blockIdx.x * 64 + lane;
  const int n_t = min(p.seq_lens[t], p.max_seq_len);
  if (static_cast<int>(blockIdx.x) * 64 >= n_t) return;
  const int c0 = t > 0 ? p.seq_query_start[t] : 0, c1 = t + 1 < p.n_seqs ? p.seq_query_start[t + 1] : p.n_queries;
  float sum = 0.f;
  for (int64_t row = static_cast<int64_t>(c0) * p.n_q_heads + wave; row < static_cast<int64_t>(c1) * p.n_q_heads; row += 4) {
    const int tok = static_cast<int>(row / p.n_q_heads), h = static_cast<int>(row % p.n_q_heads) / p.group;
    const float lse = p.lse[row];
    if (lse == -INFINITY) continue;
    stage_row<T>(p, row, q[wave], qt[wave], lane, 64);
    lds_fence();
    const int pos = p.causal ? n_t - (c1 - tok) : n_t - 1;
    const int a = min(max(p.query_adapter[p.causal ? c0 : tok], 0), p.n_adapters - 1);
    if (j < n_t && batch_sees(p, pos, j)) sum += exp2f(score<T>(p, t, j, h, a, q[wave], qt[wave]) - lse);
    lds_fence();
  }
  sum_s[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && j < n_t) {
    float* w = p.weights + t * p.weights_stride + j;
    const float all = (sum_s[0][lane] + sum_s[1][lane]) + (sum_s[2][lane] + sum_s[3][lane]);
    *w = p.decay == 0.f ? all : fmaf(p.decay, *w, all);
  }
}

template <typename T>
static hipError_t launch_weights(const WeightsParams& p, int rows, hipStream_t s) {
  if (p.b_k != nullptr) {
    const int64_t n = static_cast<int64_t>(rows) * p.rank;
    hipLaunchKernelGGL((weights_qt_kernel<T>), dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, s, p, n);
  }
  hipLaunchKernelGGL((weights_stats_kernel<T>), dim3(static_cast<unsigned>(rows < 65536 ? rows : 65536)), dim3(256), 0, s, p, static_cast<int64_t>(rows));
  hipLaunchKernelGGL((weights_sum_kernel<T>), dim3((p.max_seq_len + 63) / 64, p.n_seqs), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace lra

using namespace lra;

extern "C" {

static lra_status check_key_weights(const lra_shape* shape, const lra_cache* cache, const lra_batch* batch) {
  const lra_status st = check_batch(shape, cache, batch);
  if (st != LRA_OK) return st;
  // (a grid dimension holds fewer than 2^32 threads)
  if (cache->n_seqs > 65535 || static_cast<int64_t>(batch->n_queries) * shape->n_q_heads * shape->rank >= (int64_t{1} << 32)) return LRA_ERR_UNSUPPORTED;
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
  p.rows_per_head = batch->n_queries * p.group;
  p.row_mul = (65535 + p.group) / p.group;
  p.tile_places = pl.tile_places;
  p.weights = weights;
  p.weights_stride = weights_stride;
  p.decay = decay;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t err = pl.mfma ? launch_key_weights_mfma(p, s)
                         : shape->dtype == LRA_BF16 ? launch_weights<bf16_t>(p, pl.rows, s)
                                                    : launch_weights<float>(p, pl.rows, s);
  return err == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
