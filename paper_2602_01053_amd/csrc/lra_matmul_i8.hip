// Products of 8-bit integers with a scale per token and feature, and the quantization of their operands (contracts in lra_attn8.h).
#include "lra_attn8.h"
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

template <typename T>
__device__ __forceinline__ void load16_values(const T* src, float (&x)[16]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = reinterpret_cast<const float4*>(src)[i];
      x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(src)[i];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) x[8 * i + 2 * e] = __uint_as_float(w[e] << 16), x[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}

// One workgroup per row; sixteen values a thread and step, read twice (the second time from the caches).  8192 rows of 4096 bf16 values take
// 20.5 us, 4.9 TB/s: HBM; up to some hundred rows 2.5 to 3 us, the launch and two round trips.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantParams p) {
  __shared__ uint32_t most_s[4];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* src = static_cast<const T*>(p.x) + row * p.x_stride;
  uint32_t most = 0;
  for (int c = tid * 16; c < p.cols; c += 256 * 16) {
    float x[16];
    load16_values<T>(src + c, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), off, kWave)));
  if ((tid & 63) == 0) most_s[tid >> 6] = most;
  __syncthreads();
  most = max(max(most_s[0], most_s[1]), max(most_s[2], most_s[3]));
  const float top = __uint_as_float(most);
  const bool finite = most < 0x7f800000u;
  // (a row below 2^-119 or so: 127 / max is beyond fp32, and the largest finite factor leaves its codes smaller than they could be)
  const float inv = most == 0 || !finite ? 0.f : fminf(127.f / top, 3.402823466e38f);
  if (tid == 0) p.scales[row] = finite ? top / 127.f : __uint_as_float(0x7fc00000u);
  int8_t* dst = p.codes + row * p.codes_stride;
  for (int c = tid * 16; c < p.cols; c += 256 * 16) {
    float x[16];
    load16_values<T>(src + c, x);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[i] |= (finite ? static_cast<uint32_t>(static_cast<int>(rintf(x[4 * i + e] * inv))) & 255u : 0u) << (8 * e);
    }
    *reinterpret_cast<uint4*>(dst + c) = make_uint4(w[0], w[1], w[2], w[3]);
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

// Few tokens (32 at most): the weights are read once and nothing else counts.  A workgroup of eight waves takes 16 features and all
// tokens, a wave every eighth 64-wide piece of k, eight pieces of its weights requested at a time; operands straight from memory
// (v_mfma_i32_16x16x64_i8: a lane's 16 bytes of a row are its operand), the waves' sums meet in LDS.  RT: token tiles of 16.  4 tokens x
// 2064 features of 4096 (8.5 MB) take 5.0 us, a chain of the launch, one round trip, the exchange and the store.
template <typename T, int RT>
__global__ __launch_bounds__(512) void matmul_i8_stream_kernel(I8Params p) {
  constexpr int U = 8;
  __shared__ int sums[8][RT][4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int j0 = static_cast<int>(blockIdx.x) * 16;
  const int8_t* wr = p.w + min(j0 + l16, p.n - 1) * p.w_stride + 16 * g;
  const int8_t* xr[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) xr[rt] = p.x + min(16 * rt + l16, p.m - 1) * p.x_stride + 16 * g;
  i32x4 acc[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) acc[rt] = i32x4{0, 0, 0, 0};
  for (int c0 = wave * 64; c0 < p.k; c0 += 8 * 64 * U) {
    i32x4 a[U], b[U][RT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 512;
      const bool in = c + 16 * g < p.k;
      a[u] = in ? *reinterpret_cast<const i32x4*>(wr + c) : i32x4{0, 0, 0, 0};
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) b[u][rt] = in ? *reinterpret_cast<const i32x4*>(xr[rt] + c) : i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) acc[rt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u], b[u][rt], acc[rt], 0, 0, 0);
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][rt][e][lane] = acc[rt][e];
  __syncthreads();
  // register e: feature j0 + 4g + e of token 16 rt + l16; neighbouring threads take neighbouring features
  for (int i = threadIdx.x; i < RT * 256; i += 512) {
    const int f = i & 15, tok = i >> 4;
    if (tok >= p.m || j0 + f >= p.n) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += sums[w][tok >> 4][f & 3][(f >> 2) * 16 + (tok & 15)];
    store_scaled<T>(p, tok, j0 + f, sum);
  }
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

// 64 B features x 64 B tokens by eight waves, two of which divide k of each of the four blocks of 32 B x 32 B.  Steps of 256 / B bytes of
// k, four stages in LDS (a step's 32 KB are asked for three steps ahead: a tile is a chain of steps with nothing else to hide their
// latency).  The rows of a stage are 256 / B bytes, their 16-byte chunks exchanged by row (xor), so that sixteen rows' reads spread over
// the banks.  Bound by the way of a step's 32 KB from L2 into LDS: 0.37 us a step of B = 1 and 0.5 of B = 2, whatever the tokens: 333 tokens x
// 1056 features of 3584 9.1 us, 1024 x 4096 of 4096 24 us.  (Operands read under the products of the step before changed nothing.)
template <typename T, int B>
__global__ __launch_bounds__(512, 2) void matmul_i8_chain_kernel(I8Params p) {
  constexpr int ROWS = 64 * B, BK = 256 / B, CH = BK / 16, NS = 4, TILE = ROWS * BK, STAGE = 2 * TILE;
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
  // the second half of k is added to the first; of several blocks each half stores those of one token column
  __syncthreads();
  int* other = reinterpret_cast<int*>(smem) + (wave & 3) * (B * B * 1024) + lane;
  if constexpr (B == 1) {
    if (kh == 1) {
#pragma unroll
      for (int i = 0; i < 16; ++i) other[i * 64] = acc[0][0][i];
    }
    __syncthreads();
    if (kh == 1) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[0][0][i] += other[i * 64];
    store_block<T>(p, acc[0][0], tok0 + 32 * tb + l32, feat0 + 32 * fb, g2);
  } else {
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

// Tiles of 64, 128 or 256 a side, a compute unit holding one at a time: a round of the chip takes 10, 21 and 47 to 54 us at k = 4096, so
// that the fewest rounds by these weights are taken.  Features behind whole tiles, or behind whole rounds, may get smaller tiles in a launch of
// their own: 8192 tokens x 6160 features are 800 tiles of 256 in four rounds, 218 us, or 768 in three and 128 of 64, 188; 4096 x 4640 (of 3584)
// 304 tiles in two rounds, 96 us, or 256 in one and 160 of 128, 76.
struct I8Split {
  int side, features, rest;  // of the first launch, and the tiles' side of the other
};
static int64_t tiles_of(int64_t m, int64_t n, int64_t side) { return (m + side - 1) / side * ((n + side - 1) / side); }
static I8Split split_features(int64_t m, int64_t n) {
  auto cost = [&](int64_t features, int side) { return (tiles_of(m, features, side) + 255) / 256 * (side == 256 ? 54 : (side == 128 ? 21 : 10)); };
  I8Split best{64, static_cast<int>(n), 64};
  int64_t least = cost(n, 64);
  for (const int side : {128, 256}) {
    if (cost(n, side) < least) least = cost(n, side), best = {side, static_cast<int>(n), 64};
    const int64_t rows = (m + side - 1) / side;
    for (const int64_t columns : {n / side, tiles_of(m, n, side) / 256 * 256 / rows})
      for (const int rest : {64, 128}) {
        const int64_t first = columns * side;
        if (first <= 0 || first >= n || rest >= side) continue;
        const int64_t both = cost(first, side) + cost(n - first, rest) + 3;
        if (both < least) least = both, best = {side, static_cast<int>(first), rest};
      }
  }
  return best;
}

template <typename T>
static void launch_matmul(const I8Params& p, hipStream_t s) {
  constexpr int64_t kNear = int64_t{1} << 22;  // 256 rows within 32-bit offsets below the one that stands for "outside"
  // (up to 32 tokens while the chip holds all workgroups at once, 16 at any width: 32 tokens x 4640 features of 3584 take 15.3 us in two
  // rounds, and 8.4 us in tiles of 64; 4096 of 4096 8.4 and 9.5 us)
  if (p.m <= 16 || (p.m <= 32 && p.n <= 16 * 256)) {
    const dim3 grid((p.n + 15) / 16);
    if (p.m <= 16) hipLaunchKernelGGL((matmul_i8_stream_kernel<T, 1>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((matmul_i8_stream_kernel<T, 2>), grid, dim3(512), 0, s, p);
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
  auto grid = [](const I8Params& q, int side) { return dim3(static_cast<unsigned>((tiles_of(q.m, q.n, side) + 7) / 8 * 8)); };
  if (sp.side == 256) hipLaunchKernelGGL((matmul_i8_wide_kernel<T>), grid(first, 256), dim3(512), 0, s, first);
  else if (sp.side == 128) hipLaunchKernelGGL((matmul_i8_chain_kernel<T, 2>), grid(first, 128), dim3(512), 0, s, first);
  else hipLaunchKernelGGL((matmul_i8_chain_kernel<T, 1>), grid(first, 64), dim3(512), 0, s, first);
  if (rest.n <= 0) return;
  if (sp.rest == 128) hipLaunchKernelGGL((matmul_i8_chain_kernel<T, 2>), grid(rest, 128), dim3(512), 0, s, rest);
  else hipLaunchKernelGGL((matmul_i8_chain_kernel<T, 1>), grid(rest, 64), dim3(512), 0, s, rest);
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
