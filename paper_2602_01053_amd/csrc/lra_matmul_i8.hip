// Products of 8-bit integers with a scale per token and feature, and the quantization of their operands (contracts in lra_attn8.h).
#include "lra_attn8.h"
#include "lra_codes.h"
#include "lra_common.h"
#include "lra_prefill_util.h"

namespace lra {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct QuantParams {
  const void* x;
  int8_t* codes;
  float* scales;
  int64_t x_stride, codes_stride;
  int32_t rows, cols;
};

// Sixteen values as they lie, and as floats.
template <typename T>
struct Sixteen {
  static constexpr int N = sizeof(T);  // 16-byte pieces
  uint4 raw[N];
  __device__ __forceinline__ void load(const T* src) {
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = reinterpret_cast<const uint4*>(src)[i];
  }
  __device__ __forceinline__ void values(float (&x)[16]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) x[4 * i + e] = __uint_as_float(w[e]);
        else x[8 * i + 2 * e] = __uint_as_float(w[e] << 16), x[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    }
  }
};

// One workgroup per row; sixteen values a thread and step.  The first two steps' (8192 columns) stay in registers, what is behind them is read
// twice.  8192 rows of 4096 bf16 values take 18 to 20 us, 5.0 to 5.6 TB/s: HBM; up to some
// hundred rows 2.3 to 3.3 us, the launch and a round trip (read twice, 4 rows and their product took 9.0 us instead of 8.0).
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantParams p) {
  constexpr int KEPT = 2, STEP = 256 * 16;
  __shared__ uint32_t most_s[4];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* src = static_cast<const T*>(p.x) + row * p.x_stride;
  uint32_t most = 0;
  auto largest = [&](const Sixteen<T>& v) __attribute__((always_inline)) {
    float x[16];
    v.values(x);
#pragma unroll
    for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  };
  Sixteen<T> kept[KEPT];
#pragma unroll
  for (int k = 0; k < KEPT; ++k)
    if (k * STEP + tid * 16 < p.cols) kept[k].load(src + k * STEP + tid * 16);
#pragma unroll
  for (int k = 0; k < KEPT; ++k)
    if (k * STEP + tid * 16 < p.cols) largest(kept[k]);
  for (int c = KEPT * STEP + tid * 16; c < p.cols; c += STEP) {
    Sixteen<T> v;
    v.load(src + c);
    largest(v);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), off, kWave)));
  if ((tid & 63) == 0) most_s[tid >> 6] = most;
  __syncthreads();
  most = max(max(most_s[0], most_s[1]), max(most_s[2], most_s[3]));
  const float top = __uint_as_float(most);
  const bool finite = most < 0x7f800000u;
  // (for a largest value below 127 / (2^128 - 2^104), 3.7e-37, the factor 127 / max is beyond fp32: rows below 2^-100 are taken 2^64 times as
  // large, which rounds nothing)
  const float up = top < 0x1p-100f ? 0x1p64f : 1.f;
  const float inv = most == 0 || !finite ? 0.f : 127.f / (top * up);
  if (tid == 0) p.scales[row] = finite ? top / 127.f : __uint_as_float(0x7fc00000u);
  int8_t* dst = p.codes + row * p.codes_stride;
  auto store = [&](const Sixteen<T>& v, int c) __attribute__((always_inline)) {
    float x[16];
    v.values(x);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i] |= (finite ? static_cast<uint32_t>(static_cast<int>(rintf(x[4 * i + e] * up * inv))) & 255u : 0u) << (8 * e);
    }
    *reinterpret_cast<uint4*>(dst + c) = make_uint4(w[0], w[1], w[2], w[3]);
  };
#pragma unroll
  for (int k = 0; k < KEPT; ++k)
    if (k * STEP + tid * 16 < p.cols) store(kept[k], k * STEP + tid * 16);
  for (int c = KEPT * STEP + tid * 16; c < p.cols; c += STEP) {
    Sixteen<T> v;
    v.load(src + c);
    store(v, c);
  }
}

struct I8Params {
  const int8_t *x, *w;
  const float *x_scale, *w_scale;
  void* y;
  int64_t x_stride, w_stride, y_stride;
  int32_t m, n, k;
};

template <typename T>
__device__ __forceinline__ void store_scaled(const I8Params& p, int i, int j, int sum) {
  static_cast<T*>(p.y)[i * p.y_stride + j] = from_f32<T>(static_cast<float>(sum) * p.x_scale[i] * p.w_scale[j]);
}

// The sums' order does not matter (integers), the scaling is the same everywhere: all kernels below give the same bits.

// Few tokens (eight at most): the weights are read once and nothing else counts.  A workgroup of eight waves takes 16 features and all
// tokens, a wave every eighth 64-wide piece of k, eight pieces of its weights requested at a time; operands straight from memory
// (v_mfma_i32_16x16x64_i8: a lane's 16 bytes of a row are its operand), the waves' sums meet in LDS.  4 tokens x 2064 features of 4096
// (8.5 MB) take 4.9 us, a chain of the launch, one round trip, the exchange and the store; in tiles of 32 5.9.
template <typename T>
__global__ __launch_bounds__(512) void matmul_i8_stream_kernel(I8Params p) {
  constexpr int U = 8;
  __shared__ int sums[8][4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int j0 = static_cast<int>(blockIdx.x) * 16;
  const int8_t* wr = p.w + min(j0 + l16, p.n - 1) * p.w_stride + 16 * g;
  const int8_t* xr = p.x + min(l16, p.m - 1) * p.x_stride + 16 * g;
  i32x4 acc = {0, 0, 0, 0};
  for (int c0 = wave * 64; c0 < p.k; c0 += 8 * 64 * U) {
    i32x4 a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 512;
      const bool in = c + 16 * g < p.k;
      a[u] = in ? *reinterpret_cast<const i32x4*>(wr + c) : i32x4{0, 0, 0, 0};
      b[u] = in ? *reinterpret_cast<const i32x4*>(xr + c) : i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u], b[u], acc, 0, 0, 0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[wave][e][lane] = acc[e];
  __syncthreads();
  // register e: feature j0 + 4g + e of token l16; neighbouring threads take neighbouring features
  const int f = threadIdx.x & 15, tok = threadIdx.x >> 4;
  if (tok >= min(p.m, 16) || j0 + f >= p.n) return;
  int sum = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += sums[w][f & 3][(f >> 2) * 16 + tok];
  store_scaled<T>(p, tok, j0 + f, sum);
}

// The scaled sums of a 32 x 32 block: register i of a lane is feature f0 + 8 (i / 4) + 4 g2 + i % 4 of token `tok`.
typedef int i32x16 __attribute__((ext_vector_type(16)));
template <typename T>
__device__ __forceinline__ void store_block(const I8Params& p, const i32x16& acc, int tok, int f0, int g2) {
  if (tok >= p.m) return;
  const float xs = p.x_scale[tok];
  T* row = static_cast<T*>(p.y) + tok * p.y_stride;
  const bool whole = (p.y_stride & 3) == 0;  // (four features lie together and aligned)
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int f = f0 + 8 * q + 4 * g2;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(acc[4 * q + e]) * xs * p.w_scale[min(f + e, p.n - 1)];
    if (whole && f + 4 <= p.n) {
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(row + f) = make_uint2(pf_pack2(v[0], v[1]), pf_pack2(v[2], v[3]));
      else *reinterpret_cast<float4*>(row + f) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (f + e < p.n) row[f + e] = from_f32<T>(v[e]);
    }
  }
}

// A wave's A x B blocks in bf16, rows of y 16 bytes aligned: through its part of LDS, from where they go out in rows of 64 A bytes (a
// lane's registers are one token's features, 16 bytes of a row beside each other; stored from there, 8192 tokens x 4096 features of 4096 took
// 134 us instead of 122).  A token's 16-byte chunks are exchanged (xor), so that sixteen tokens' accesses spread over the banks.
template <int A, int B, typename F>
__device__ __forceinline__ void store_by_rows(const I8Params& p, unsigned char* mine, int tok0, int feat0, int lane, F block) {
  constexpr int CH = 4 * A, ROW = 64 * A;
  static_assert(CH == 16 || CH == 8);
  const int l32 = lane & 31, g2 = lane >> 5;
  auto place = [](int tok, int c) __attribute__((always_inline)) -> int { return tok * ROW + ((c ^ (CH == 16 ? tok & 15 : (tok >> 1) & 7)) << 4); };
#pragma unroll
  for (int b = 0; b < B; ++b) {
    const int tok = 32 * b + l32;
    const float xs = p.x_scale[min(tok0 + tok, p.m - 1)];
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(block(a, b)[4 * q + e]) * xs * p.w_scale[min(feat0 + 32 * a + 8 * q + 4 * g2 + e, p.n - 1)];
        *reinterpret_cast<uint2*>(mine + place(tok, 4 * a + q) + 8 * g2) = make_uint2(pf_pack2(v[0], v[1]), pf_pack2(v[2], v[3]));
      }
  }
  wave_fence();
  const int c = lane % CH, f = feat0 + 8 * c;
#pragma unroll
  for (int i = 0; i < 32 * B * CH / 64; ++i) {
    const int tok = (64 / CH) * i + lane / CH;
    const uint4 v = *reinterpret_cast<const uint4*>(mine + place(tok, c));
    if (tok0 + tok >= p.m) continue;
    bf16_t* const at = static_cast<bf16_t*>(p.y) + (tok0 + tok) * p.y_stride + f;
    if (f + 8 <= p.n) {
      *reinterpret_cast<uint4*>(at) = v;
    } else {
      const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (f + e < p.n) at[e] = static_cast<bf16_t>(x[e >> 1] >> (16 * (e & 1)));
    }
  }
}

// Workgroup -> tile.  Consecutive workgroups go to consecutive XCDs: an XCD takes an eighth of the tiles, one after the other, token
// tiles in fours and the feature tiles of a four in turn, so that what it works on at a time shares its L2.
__device__ __forceinline__ bool tile_of(int n_tt, int n_ct, int& tt, int& ct) {
  const int total = n_tt * n_ct, per = (total + 7) / 8;
  const int i = static_cast<int>(blockIdx.x) >> 3, tile = (static_cast<int>(blockIdx.x) & 7) * per + i;
  if (i >= per || tile >= total) return false;
  const int grp = tile / (4 * n_ct), r = tile - grp * 4 * n_ct, high = min(4, n_tt - 4 * grp);
  ct = r / high;
  tt = 4 * grp + r - ct * high;
  return true;
}

// 32 FB features x 32 TB tokens by eight waves, 8 / (FB TB) of which divide k of each of the 32 x 32 blocks.  Steps of 256 bytes of k, four
// stages in LDS (a step's tiles are asked for three steps ahead: a workgroup is a chain of steps with nothing else to hide their latency).
// A row of a stage is 256 bytes, its 16-byte chunks exchanged by row (xor), so that sixteen rows' reads spread over the banks.  Bound by
// the way of a step's 8 (FB + TB) KB from L2 into LDS, whatever the tokens (five stages changed nothing), so the smaller the tiles the shorter the chain, as long as
// the chip holds them: 64 tokens x 4096 features of 4096 take 6.0 us in tiles of 32, 7.4 of 64 x 32 and 9.5 of 64; 128 tokens 8.7, 7.8 and 9.5;
// 256 tokens 15.9, 14 and 10.4.
template <typename T, int FB, int TB>
__global__ __launch_bounds__(512, 2) void matmul_i8_small_kernel(I8Params p) {
  constexpr int BK = 256, NS = 4, W_TILE = 32 * FB * BK, STAGE = W_TILE + 32 * TB * BK, NB = FB * TB, KG = 8 / NB, KS = 8 / KG;
  constexpr int SUMS = 8 * 1024 * 4;
  __shared__ __align__(16) unsigned char smem[NS * STAGE > SUMS ? NS * STAGE : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, g2 = lane >> 5;
  int tt, ct;
  if (!tile_of((p.m + 32 * TB - 1) / (32 * TB), (p.n + 32 * FB - 1) / (32 * FB), tt, ct)) return;
  const int tok0 = tt * 32 * TB, feat0 = ct * 32 * FB;
  const uint32_t ldw = static_cast<uint32_t>(p.w_stride), ldx = static_cast<uint32_t>(p.x_stride);  // (at most 2^22)
  const pf_u32x4 rs_w = pf_rsrc(p.w + feat0 * p.w_stride, (min(32 * FB, p.n - feat0) - 1u) * ldw + p.k);
  const pf_u32x4 rs_x = pf_rsrc(p.x + tok0 * p.x_stride, (min(32 * TB, p.m - tok0) - 1u) * ldx + p.k);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem)));
  // request i of eight per 32 rows fills rows 4i .. 4i + 3; wave w has i = w of each 32
  const int row = 4 * wave + (lane >> 4), chunk = (lane & 15) ^ (row & 15);
  const int n_steps = (p.k + BK - 1) / BK;
  auto issue = [&](int step) __attribute__((always_inline)) {
    const bool in = step * BK + chunk * 16 < p.k;  // (behind the last column: zeros)
    const uint32_t dst = lds0 + (step % NS) * STAGE + wave * 1024;
#pragma unroll
    for (int q = 0; q < FB; ++q) pf_load16_to_lds(rs_w, dst + q * 32 * BK, in ? (row + 32u * q) * ldw + chunk * 16 : kPfOob, step * BK);
#pragma unroll
    for (int q = 0; q < TB; ++q) pf_load16_to_lds(rs_x, dst + W_TILE + q * 32 * BK, in ? (row + 32u * q) * ldx + chunk * 16 : kPfOob, step * BK);
  };
  for (int s = 0; s < NS - 1; ++s)
    if (s < n_steps) issue(s);
  const int blk = wave % NB, kg = wave / NB, fb = blk % FB, tb = blk / FB;
  const int a_row = (32 * fb + l32) * BK, b_row = W_TILE + (32 * tb + l32) * BK, swap = l32 & 15;
  i32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0;
  for (int s = 0; s < n_steps; ++s) {
    // this step's requests of the wave are here, those of the two behind it may be on their way
    if (s + 2 < n_steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (FB + TB)));
    else if (s + 1 < n_steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(FB + TB));
    else pf_wait_vm0();
    __syncthreads();  // ... and everybody's; and everybody has read the stage that is filled next
    if (s + NS - 1 < n_steps) issue(s + NS - 1);
    const unsigned char* st = smem + (s % NS) * STAGE;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int c = ((2 * (KS * kg + ks) + g2) ^ swap) << 4;
      const i32x4 a = *reinterpret_cast<const i32x4*>(st + a_row + c), b = *reinterpret_cast<const i32x4*>(st + b_row + c);
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
  }
  // the waves of a block meet in LDS, each of them adds up and stores its part of the registers: register i of a lane is feature
  // 8 (i / 4) + 4 g2 + i % 4 of its token
  constexpr int R = 16 / KG, V = R < 4 ? R : 4;
  __syncthreads();
  int* const sums = reinterpret_cast<int*>(smem) + blk * 1024 + lane;
#pragma unroll
  for (int i = 0; i < 16; ++i) sums[kg * NB * 1024 + i * 64] = acc[i];
  __syncthreads();
  const int tok = tok0 + 32 * tb + l32;
  if (tok >= p.m) return;
  const float xs = p.x_scale[tok];
  T* const out = static_cast<T*>(p.y) + tok * p.y_stride;
  const bool whole = p.y_stride % V == 0;  // (V features lie together and aligned)
#pragma unroll
  for (int o = 0; o < R; o += V) {
    const int i0 = R * kg + o, f = feat0 + 32 * fb + 8 * (i0 >> 2) + 4 * g2 + (i0 & 3);
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      int sum = 0;
#pragma unroll
      for (int g = 0; g < KG; ++g) sum += sums[g * NB * 1024 + (i0 + e) * 64];
      v[e] = static_cast<float>(sum) * xs * p.w_scale[min(f + e, p.n - 1)];
    }
    if (whole && f + V <= p.n) {
      if constexpr (V == 4 && sizeof(T) == 2) *reinterpret_cast<uint2*>(out + f) = make_uint2(pf_pack2(v[0], v[1]), pf_pack2(v[2], v[3]));
      else if constexpr (V == 4) *reinterpret_cast<float4*>(out + f) = make_float4(v[0], v[1], v[2], v[3]);
      else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(out + f) = pf_pack2(v[0], v[1]);
      else *reinterpret_cast<float2*>(out + f) = make_float2(v[0], v[1]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (f + e < p.n) out[f + e] = from_f32<T>(v[e]);
    }
  }
}

// 128 features x 128 tokens by eight waves, two of which divide k of each of the four blocks of 64 x 64.  As above, in steps of 128 bytes and
// with the same bound, 0.5 us a step: 1024 tokens x 4096 features of 4096 24 us.  (Operands read under the products of the step before
// changed nothing.)
template <typename T>
__global__ __launch_bounds__(512, 2) void matmul_i8_chain_kernel(I8Params p) {
  constexpr int B = 2, ROWS = 64 * B, BK = 256 / B, CH = BK / 16, NS = 4, TILE = ROWS * BK, STAGE = 2 * TILE;
  __shared__ __align__(16) unsigned char smem[NS * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, g2 = lane >> 5;
  int tt, ct;
  if (!tile_of((p.m + ROWS - 1) / ROWS, (p.n + ROWS - 1) / ROWS, tt, ct)) return;
  const int tok0 = tt * ROWS, feat0 = ct * ROWS;
  const uint32_t ldw = static_cast<uint32_t>(p.w_stride), ldx = static_cast<uint32_t>(p.x_stride);  // (at most 2^22)
  const pf_u32x4 rs_w = pf_rsrc(p.w + feat0 * p.w_stride, (min(ROWS, p.n - feat0) - 1u) * ldw + p.k);
  const pf_u32x4 rs_x = pf_rsrc(p.x + tok0 * p.x_stride, (min(ROWS, p.m - tok0) - 1u) * ldx + p.k);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem)));
  // request i of sixteen per tile fills rows 4 B i .. 4 B i + 4 B - 1; wave w has i = w and w + 8; row r's chunk c is at c ^ (r / B) % CH
  const int row = lane / CH, chunk = (lane & (CH - 1)) ^ ((4 * wave + row / B) & (CH - 1));
  const int n_steps = (p.k + BK - 1) / BK;
  auto issue = [&](int step) __attribute__((always_inline)) {
    const bool in = step * BK + chunk * 16 < p.k;  // (behind the last column: zeros)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int r = 4 * B * (wave + 8 * q) + row;
      const uint32_t dst = lds0 + (step % NS) * STAGE + (wave + 8 * q) * 1024;
      pf_load16_to_lds(rs_w, dst, in ? r * ldw + chunk * 16 : kPfOob, step * BK);
      pf_load16_to_lds(rs_x, dst + TILE, in ? r * ldx + chunk * 16 : kPfOob, step * BK);
    }
  };
  for (int s = 0; s < NS - 1; ++s)
    if (s < n_steps) issue(s);
  const int kh = wave >> 2, fb = wave & 1, tb = (wave >> 1) & 1;
  const int a_row = (32 * B * fb + l32) * BK, b_row = TILE + (32 * B * tb + l32) * BK, swap = (l32 / B) & (CH - 1);
  i32x16 acc[B][B];
#pragma unroll
  for (int a = 0; a < B; ++a)
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0;
  for (int s = 0; s < n_steps; ++s) {
    // this step's four requests of the wave are here, those of the two behind it may be on their way
    if (s + 2 < n_steps) asm volatile("s_waitcnt vmcnt(8)");
    else if (s + 1 < n_steps) asm volatile("s_waitcnt vmcnt(4)");
    else pf_wait_vm0();
    __syncthreads();  // ... and everybody's; and everybody has read the stage that is filled next
    if (s + NS - 1 < n_steps) issue(s + NS - 1);
    const unsigned char* st = smem + (s % NS) * STAGE;
#pragma unroll
    for (int ks = 0; ks < BK / 64; ++ks) {
      const int c = ((CH / 2 * kh + 2 * ks + g2) ^ swap) << 4;
      i32x4 a[B], b[B];
#pragma unroll
      for (int i = 0; i < B; ++i) {
        a[i] = *reinterpret_cast<const i32x4*>(st + a_row + i * 32 * BK + c);
        b[i] = *reinterpret_cast<const i32x4*>(st + b_row + i * 32 * BK + c);
      }
#pragma unroll
      for (int i = 0; i < B; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    }
  }
  // each half of k has the sums of one token column of its blocks from the other
  __syncthreads();
  int* other = reinterpret_cast<int*>(smem) + (wave & 3) * (B * B * 1024) + lane;
#pragma unroll
  for (int a = 0; a < B; ++a)
#pragma unroll
    for (int i = 0; i < 16; ++i) other[((kh ^ 1) * B + a) * 1024 + i * 64] = kh ? acc[a][0][i] : acc[a][1][i];
  __syncthreads();
  i32x16 sum[B];
#pragma unroll
  for (int a = 0; a < B; ++a)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[a][i] = (kh ? acc[a][1][i] : acc[a][0][i]) + other[(kh * B + a) * 1024 + i * 64];
  const int tok = tok0 + 32 * (B * tb + kh), f0 = feat0 + 32 * B * fb;
  if constexpr (sizeof(T) == 2) {
    if ((p.y_stride & 7) == 0) {
      store_by_rows<B, 1>(p, smem + 4 * B * B * 4096 + wave * B * 2048, tok, f0, lane, [&](int a, int) -> const i32x16& { return sum[a]; });
      return;
    }
  }
#pragma unroll
  for (int a = 0; a < B; ++a)
    if (f0 + 32 * a < p.n) store_block<T>(p, sum[a], tok + l32, f0 + 32 * a, g2);
}

// 256 features x 256 tokens by eight waves of 128 x 64 (eight 32 x 32 accumulators): six operand reads for eight products, 64 KB into
// LDS for 16.8 M multiply-adds.  Steps of 128 bytes of k, two stages, one workgroup per compute unit; the two waves of a SIMD cover each
// other's reads and requests.  Bound by the matrix cores at the clock that they leave (busy 54 %) and the steps' 64 KB from L2: 4096 tokens x
// 4096 features of 4096 63 us, 2.2 POP/s; 8192 x 14336 407, 2.4; a round of 256 tiles takes 47 to 54.  (Steps of 64 bytes in four stages: a
// sixth longer, rows in pieces of half a line.)
template <typename T>
__global__ __launch_bounds__(512, 2) void matmul_i8_wide_kernel(I8Params p) {
  constexpr int BK = 128, TILE = 256 * BK, STAGE = 2 * TILE;
  __shared__ __align__(16) unsigned char smem[2 * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, g2 = lane >> 5;
  const int wr = wave >> 2, wc = wave & 3;
  int tt, ct;
  if (!tile_of((p.m + 255) / 256, (p.n + 255) / 256, tt, ct)) return;
  const int tok0 = tt * 256, feat0 = ct * 256;
  const uint32_t ldw = static_cast<uint32_t>(p.w_stride), ldx = static_cast<uint32_t>(p.x_stride);  // (at most 2^22)
  const pf_u32x4 rs_w = pf_rsrc(p.w + feat0 * p.w_stride, (min(256, p.n - feat0) - 1u) * ldw + p.k);
  const pf_u32x4 rs_x = pf_rsrc(p.x + tok0 * p.x_stride, (min(256, p.m - tok0) - 1u) * ldx + p.k);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(PF_LDS_AS(unsigned char, smem)));
  // request i of thirty-two per tile fills rows 8i .. 8i + 7, wave w has i = w + 8 part; chunk c of row r at c ^ (r / 2) % 8
  const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
  // (rows by the lanes' offsets: what a resource's size cuts does not hang on how it counts the scalar one)
  uint32_t w_off[4], x_off[4];
#pragma unroll
  for (int part = 0; part < 4; ++part) {
    const uint32_t row = 8u * (wave + 8 * part) + (lane >> 3);
    w_off[part] = row * ldw + chunk * 16, x_off[part] = row * ldx + chunk * 16;
  }
  auto issue = [&](int step, int st, int part) __attribute__((always_inline)) {
    const uint32_t dst = lds0 + st * STAGE + (wave + 8 * part) * 1024;
    const bool in = step * BK + chunk * 16 < p.k;  // (behind the last column: zeros)
    pf_load16_to_lds(rs_w, dst, in ? w_off[part] : kPfOob, step * BK);
    pf_load16_to_lds(rs_x, dst + TILE, in ? x_off[part] : kPfOob, step * BK);
  };
  const int n_steps = (p.k + BK - 1) / BK;
#pragma unroll
  for (int part = 0; part < 4; ++part) issue(0, 0, part);
  const int pre = l32 * BK + (((l32 >> 1) & 7) << 4);
  const int fbase = 4 * wr, tbase = 2 * wc;
  i32x16 acc[4][2];
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0;
  // the tiles have landed, everybody is done with the other stage; the requests of the next step go out beside the products of the first
  // two slices, the operands of a slice are read under the products of the one before
  auto k_step = [&](int step, auto st_c, bool more) __attribute__((always_inline)) {
    constexpr int ST = decltype(st_c)::value;
    constexpr int KS = BK / 32;
    pf_wait_vm0();
    __syncthreads();
    const unsigned char* wt = smem + ST * STAGE + fbase * 32 * BK;
    const unsigned char* xt = smem + ST * STAGE + TILE + tbase * 32 * BK;
    i32x4 a[2][4], b[2][2];
    auto read_slice = [&](int ks, int buf) __attribute__((always_inline)) {
      const int off = pre ^ ((2 * ks + g2) << 4);
#pragma unroll
      for (int j = 0; j < 2; ++j) b[buf][j] = *reinterpret_cast<const i32x4*>(xt + off + j * 32 * BK);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[buf][i] = *reinterpret_cast<const i32x4*>(wt + off + i * 32 * BK);
    };
    read_slice(0, 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int cur = ks & 1;
      __builtin_amdgcn_sched_barrier(0);
      if (more && ks < 2) {
        issue(step + 1, ST ^ 1, 2 * ks);
        issue(step + 1, ST ^ 1, 2 * ks + 1);
      }
      if (ks + 1 < KS) read_slice(ks + 1, cur ^ 1);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[cur][i], b[cur][j], acc[i][j], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int step = 0; step < n_steps; step += 2) {
    k_step(step, std::integral_constant<int, 0>{}, step + 1 < n_steps);
    if (step + 1 < n_steps) k_step(step + 1, std::integral_constant<int, 1>{}, step + 2 < n_steps);
  }
  if constexpr (sizeof(T) == 2) {
    if ((p.y_stride & 7) == 0) {
      __syncthreads();
      store_by_rows<4, 2>(p, smem + wave * 16384, tok0 + 32 * tbase, feat0 + 32 * fbase, lane, [&](int a, int b) -> const i32x16& { return acc[a][b]; });
      return;
    }
  }
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int f0 = feat0 + 32 * (fbase + a);
      if (f0 < p.n) store_block<T>(p, acc[a][b], tok0 + 32 * (tbase + b) + l32, f0, g2);
    }
}

// Rows too far apart for the other kernels' offsets: a wave per 16 features and 16 tokens, operands straight from memory.
template <typename T>
__global__ __launch_bounds__(256) void matmul_i8_far_kernel(I8Params p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int j0 = (static_cast<int>(blockIdx.x) * 4 + wave) * 16;
  if (j0 >= p.n) return;
  const int8_t* wr = p.w + min(j0 + l16, p.n - 1) * p.w_stride + 16 * g;
  for (int i0 = static_cast<int>(blockIdx.y) * 16; i0 < p.m; i0 += gridDim.y * 16) {
    const int8_t* xr = p.x + min(i0 + l16, p.m - 1) * p.x_stride + 16 * g;
    i32x4 acc = {0, 0, 0, 0};
    for (int c = 0; c < p.k; c += 64) {
      i32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
      if (c + 16 * g < p.k) {
        a = *reinterpret_cast<const i32x4*>(wr + c);
        b = *reinterpret_cast<const i32x4*>(xr + c);
      }
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc, 0, 0, 0);
    }
    const int i = i0 + l16;
    if (i >= p.m) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j0 + 4 * g + e < p.n) store_scaled<T>(p, i, j0 + 4 * g + e, acc[e]);
  }
}

// Tiles of 32 to 256 a side by what they cost: a launch and the rounds of the chip that it takes, a compute unit holding one tile at a
// time (two of 32, which the figures count as two rounds of half the length).  Features behind whole tiles, or behind whole rounds,
// may get smaller tiles in a launch of their own: 8192 tokens x 6160 features are 800 tiles of 256 in four rounds, 218 us, or 768 in
// three and a few small ones, 188; 4096 x 4640 (of 3584) 304 tiles in two rounds, 96 us, or 256 in one and 160 of 128, 76.  (The figures are those of
// k = 4096 for any k: of short rows a second launch may cost what it saves.)
enum I8Tile { kTile32, kTile64x32, kTile32x64, kTile64, kTile128, kTile256 };  // features x tokens
struct I8Shape {
  int features, tokens, start, round;  // time of a launch and of each round of the chip, in 0.1 us at k = 4096
};
constexpr I8Shape kI8Shapes[] = {{32, 32, 24, 32}, {64, 32, 8, 64}, {32, 64, 8, 64}, {64, 64, 5, 88}, {128, 128, 0, 210}, {256, 256, 0, 540}};
struct I8Split {
  int tile, features, rest;  // of the first launch, and the tile of the other
};
static int64_t tiles_of(int64_t m, int64_t n, int tile) {
  const I8Shape& s = kI8Shapes[tile];
  return (m + s.tokens - 1) / s.tokens * ((n + s.features - 1) / s.features);
}
static I8Split split_features(int64_t m, int64_t n) {
  auto cost = [&](int64_t features, int tile) { return kI8Shapes[tile].start + (tiles_of(m, features, tile) + 255) / 256 * kI8Shapes[tile].round; };
  I8Split best{kTile64, static_cast<int>(n), kTile64};
  int64_t least = cost(n, kTile64);
  for (int tile = kTile32; tile <= kTile256; ++tile) {
    if (cost(n, tile) < least) least = cost(n, tile), best = {tile, static_cast<int>(n), kTile64};
    if (tile < kTile128) continue;
    const int64_t side = kI8Shapes[tile].features, rows = (m + side - 1) / side;
    for (const int64_t columns : {n / side, tiles_of(m, n, tile) / 256 * 256 / rows})
      for (int rest = kTile32; rest < tile; ++rest) {
        const int64_t first = columns * side;
        if (first <= 0 || first >= n) continue;
        const int64_t both = cost(first, tile) + cost(n - first, rest) + 30;
        if (both < least) least = both, best = {tile, static_cast<int>(first), rest};
      }
  }
  return best;
}

template <typename T>
static void launch_tiles(const I8Params& p, int tile, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((tiles_of(p.m, p.n, tile) + 7) / 8 * 8));
  switch (tile) {
    case kTile32: hipLaunchKernelGGL((matmul_i8_small_kernel<T, 1, 1>), grid, dim3(512), 0, s, p); break;
    case kTile64x32: hipLaunchKernelGGL((matmul_i8_small_kernel<T, 2, 1>), grid, dim3(512), 0, s, p); break;
    case kTile32x64: hipLaunchKernelGGL((matmul_i8_small_kernel<T, 1, 2>), grid, dim3(512), 0, s, p); break;
    case kTile64: hipLaunchKernelGGL((matmul_i8_small_kernel<T, 2, 2>), grid, dim3(512), 0, s, p); break;
    case kTile128: hipLaunchKernelGGL((matmul_i8_chain_kernel<T>), grid, dim3(512), 0, s, p); break;
    default: hipLaunchKernelGGL((matmul_i8_wide_kernel<T>), grid, dim3(512), 0, s, p);
  }
}

template <typename T>
static void launch_matmul(const I8Params& p, hipStream_t s) {
  constexpr int64_t kNear = int64_t{1} << 22;  // 256 rows within 32-bit offsets below the one that stands for "outside"
  // (while the chip holds all workgroups at once: 4 tokens x 6160 features of 4096 take 8.1 us in two rounds, in tiles of 32 6.6; of 4096
  // features 5.6 and 6.0; 16 tokens x 4096 6.4 and 6.0)
  if (p.m <= 8 && p.n <= 16 * 256) {
    hipLaunchKernelGGL((matmul_i8_stream_kernel<T>), dim3((p.n + 15) / 16), dim3(512), 0, s, p);
    return;
  }
  if (p.x_stride > kNear || p.w_stride > kNear) {
    hipLaunchKernelGGL((matmul_i8_far_kernel<T>), dim3((p.n + 63) / 64, min((p.m + 15) / 16, 65535)), dim3(256), 0, s, p);
    return;
  }
  const I8Split sp = split_features(p.m, p.n);
  I8Params first = p, rest = p;
  first.n = sp.features;
  rest.n = p.n - sp.features;
  rest.w += sp.features * p.w_stride;
  rest.w_scale += sp.features;
  rest.y = static_cast<T*>(p.y) + sp.features;
  launch_tiles<T>(first, sp.tile, s);
  if (rest.n > 0) launch_tiles<T>(rest, sp.rest, s);
}

}  // namespace lra

using namespace lra;

extern "C" {

lra_status lra_quantize_rows(const void* x, int32_t dtype, int64_t x_stride, int32_t rows, int32_t cols, int8_t* codes,
                             int64_t codes_stride, float* scales, void* stream) {
  if (!x || !codes || !scales) return LRA_ERR_NULL;
  if (dtype != LRA_BF16 && dtype != LRA_F32) return LRA_ERR_DTYPE;
  const int64_t es = dtype == LRA_BF16 ? 2 : 4;
  if (rows < 1 || cols < 1 || x_stride < cols || codes_stride < cols) return LRA_ERR_SHAPE;
  if (cols % 16 || cols > (1 << 17) || rows >= (1 << 24) || x_stride > (int64_t{1} << 40) || codes_stride > (int64_t{1} << 40)) return LRA_ERR_UNSUPPORTED;
  if (((x_stride * es) | codes_stride) & 15) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(codes)) & 15 || reinterpret_cast<uintptr_t>(scales) & 3) return LRA_ERR_SHAPE;
  const QuantParams p{x, codes, scales, x_stride, codes_stride, rows, cols};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == LRA_BF16) hipLaunchKernelGGL((quantize_rows_kernel<bf16_t>), dim3(rows), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((quantize_rows_kernel<float>), dim3(rows), dim3(256), 0, s, p);
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

static lra_status check_i8_sizes(int32_t m, int32_t n, int32_t k, int32_t dtype) {
  if (dtype != LRA_BF16 && dtype != LRA_F32) return LRA_ERR_DTYPE;
  if (m < 1 || n < 1 || k < 1) return LRA_ERR_SHAPE;
  if (k % 16 || k >= (1 << 17) || m > (1 << 20) || n > (1 << 20)) return LRA_ERR_UNSUPPORTED;
  return LRA_OK;
}

size_t lra_matmul_i8_workspace_bytes(int32_t m, int32_t n, int32_t k, int32_t dtype) {
  if (check_i8_sizes(m, n, k, dtype) != LRA_OK) return static_cast<size_t>(-1);
  return 0;
}

lra_status lra_matmul_i8(const lra_i8_operands* ops, void* y, int32_t dtype, int64_t y_stride, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (!ops || !y || !ops->x || !ops->w || !ops->x_scale || !ops->w_scale) return LRA_ERR_NULL;
  const lra_status st = check_i8_sizes(ops->m, ops->n, ops->k, dtype);
  if (st != LRA_OK) return st;
  if (ops->x_stride < ops->k || ops->w_stride < ops->k || y_stride < ops->n) return LRA_ERR_SHAPE;
  if (ops->x_stride > (int64_t{1} << 31) || ops->w_stride > (int64_t{1} << 31) || y_stride > (int64_t{1} << 31)) return LRA_ERR_UNSUPPORTED;
  if ((ops->x_stride | ops->w_stride) & 15) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(ops->x) | reinterpret_cast<uintptr_t>(ops->w) | reinterpret_cast<uintptr_t>(y)) & 15) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(ops->x_scale) | reinterpret_cast<uintptr_t>(ops->w_scale)) & 3) return LRA_ERR_SHAPE;
  (void)workspace, (void)workspace_bytes;
  const I8Params p{ops->x, ops->w, ops->x_scale, ops->w_scale, y, ops->x_stride, ops->w_stride, y_stride, ops->m, ops->n, ops->k};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == LRA_BF16) launch_matmul<bf16_t>(p, s);
  else launch_matmul<float>(p, s);
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
