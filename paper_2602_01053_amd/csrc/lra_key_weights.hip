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

__device__ __forceinline__ float quad_sum(float v) {  // over four neighbouring lanes, in each of them
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xb1, 0xf, 0xf, false));  // [1,0,3,2]
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4e, 0xf, 0xf, false));  // [2,3,0,1]
}

// scale log2(e) times the score of a row (q and Qt in LDS) and this lane's key, number 16 (lane % 4) + lane / 4 of the wave's 64;
// token(i) is the i-th of them, -1 for none (it is not read; any score comes back).  Four lanes share a row's 16-byte pieces, so that
// a load touches sixteen rows and not 64, and four keys one after another.  (A key per lane: the call for 4 queries of 30000 fp32 tokens,
// 32 heads of 128, 676 us against 296; 40 queries of 8000, 8 heads of 64, 461 against 156; rank 12 in bf16, 30000 tokens, 354 against 261.)
template <typename T, int D, typename F>
__device__ __forceinline__ float score(const WeightsParams& p, int t, int h, int a, const float* q, const float* qt, F token) {
  constexpr int E = 16 / static_cast<int>(sizeof(T)), N = D / E / 4;  // pieces of a lane
  constexpr int KEYS = E == 8 && D == 128 ? 1 : 8 / N;                // requested together (bf16 at d = 128: registers for one)
  const int lane = threadIdx.x & 63, part = lane & 3;
  float own = 0.f;
#pragma unroll
  for (int g0 = 0; g0 < 4; g0 += KEYS) {
    u32x4 v[KEYS][N];
    const T* l[KEYS];
    bool any[KEYS];
#pragma unroll
    for (int g = 0; g < KEYS; ++g) {
      const int j = token(16 * (g0 + g) + (lane >> 2));
      any[g] = j >= 0;
#pragma unroll
      for (int c = 0; c < N; ++c) v[g][c] = u32x4{0u, 0u, 0u, 0u};
      l[g] = static_cast<const T*>(p.l);
      if (any[g]) {
        const u32x4* k = reinterpret_cast<const u32x4*>(static_cast<const T*>(p.k_base) + kv_offset(p, t, j, h));
#pragma unroll
        for (int c = 0; c < N; ++c) v[g][c] = k[4 * c + part];
        l[g] += l_offset(p, t, j, a);
      }
    }
    float acc[KEYS];
#pragma unroll
    for (int g = 0; g < KEYS; ++g) acc[g] = 0.f;
    if (p.b_k != nullptr) {
      for (int r0 = part; r0 < p.rank; r0 += 16) {
        T x[KEYS][4];
#pragma unroll
        for (int g = 0; g < KEYS; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[g][e] = any[g] && r0 + 4 * e < p.rank ? l[g][r0 + 4 * e] : T{};
#pragma unroll
        for (int g = 0; g < KEYS; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[g] = fmaf(to_f32<T>(x[g][e]), qt[min(r0 + 4 * e, 63)], acc[g]);
      }
    }
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float qe = q[(4 * c + part) * E + e];
#pragma unroll
        for (int g = 0; g < KEYS; ++g) {
          float x;
          if constexpr (sizeof(T) == 4) x = __uint_as_float(v[g][c][e]);
          else x = __uint_as_float((e & 1) ? (v[g][c][e >> 1] & 0xffff0000u) : (v[g][c][e >> 1] << 16));
          acc[g] = fmaf(x, qe, acc[g]);
        }
      }
#pragma unroll
    for (int g = 0; g < KEYS; ++g) {
      const float s = quad_sum(acc[g]);
      own = part == g0 + g ? s : own;
    }
    if constexpr (D == 128) __builtin_amdgcn_sched_barrier(0);  // (the rows of further keys in flight would need scratch memory)
  }
  return own * (p.scale * kLog2e);
}

// One workgroup per row and key share; a wave takes 64 keys of every 256.  Qt of the row is formed here, four lanes to a rank, and left
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
    const int own = 16 * (tid & 3) + ((tid & 63) >> 2);
    for (int k = static_cast<int>(static_cast<int64_t>(b.n_keys) * split / p.n_splits) + (tid & ~63); k < k1; k += 256) {
      float s = score<T, D>(p, b.t, h, b.adapter, q, qt, [&](int i) { return k + i >= k1 ? -1 : (k + i < b.n_sinks ? k + i : k + i + b.gap); });
      if (k + own >= k1) s = -INFINITY;
      if (tile_reference(s) == -INFINITY) continue;
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
  const int j0 = blockIdx.x * 64, own = 16 * (lane & 3) + (lane >> 2);  // the lane's key: j0 + own
  const int n_t = min(p.seq_lens[t], p.max_seq_len);
  if (static_cast<int>(blockIdx.x) * 64 >= n_t) return;
  const int c0 = t > 0 ? p.seq_query_start[t] : 0, c1 = t + 1 < p.n_seqs ? p.seq_query_start[t + 1] : p.n_queries;
  float sum = 0.f;
  for (int64_t row = static_cast<int64_t>(c0) * p.n_q_heads + wave; row < static_cast<int64_t>(c1) * p.n_q_heads; row += 16) {
    const int tok = static_cast<int>(row / p.n_q_heads), h = static_cast<int>(row % p.n_q_heads) / p.group;
    const float2 ml = lane < p.n_splits ? reinterpret_cast<const float2*>(p.stats)[row * p.n_splits + lane] : make_float2(-INFINITY, 0.f);
    for (int c = lane; c < D; c += 64) q[wave][c] = to_f32<T>(static_cast<const T*>(p.q)[row * D + c]);
    qt[wave][lane] = p.b_k != nullptr && lane < p.rank ? p.qt[row * p.rank + lane] : 0.f;
    lds_fence();
    const int pos = p.causal ? n_t - (c1 - tok) : n_t - 1;
    const int a = min(max(p.query_adapter[p.causal ? c0 : tok], 0), p.n_adapters - 1);
    auto seen = [&](int i) { return j0 + i < n_t && batch_sees(p, pos, j0 + i); };
    const float s = score<T, D>(p, t, h, a, q[wave], qt[wave], [&](int i) { return seen(i) ? j0 + i : -1; });
    lds_fence();
    // the shares' statistics joined, a lane each (32 at most), while the key's row is on its way
    const float top = wave_max(ml.x);
    const float all = wave_sum(ml.x == -INFINITY ? ml.y : ml.y * exp2f(ml.x - top));  // (a share's NaN is the row's)
    if (all != 0.f && seen(own)) sum += exp2f(s - (top + log2f(all)));  // (0: the row sees nothing)
  }
  sum_s[wave][own] = sum;
  __syncthreads();
  if (wave == 0 && j0 + lane < n_t) {
    float* w = p.weights + t * p.weights_stride + j0 + lane;
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
  // (sequences in a grid's y; sixteen threads per token in a dimension of fewer than 2^32)
  if (cache->n_seqs > 65535 || cache->max_seq_len > (1 << 27)) return LRA_ERR_UNSUPPORTED;
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
