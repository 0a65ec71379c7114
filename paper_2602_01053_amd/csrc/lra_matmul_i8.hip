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

// One workgroup per row; sixteen values a thread and step, read twice.
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

// A wave per 16 features and 16 tokens: W x^T by v_mfma_i32_16x16x64_i8, operands straight from memory.
template <typename T>
__global__ __launch_bounds__(256) void matmul_i8_kernel(I8Params p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int j0 = (static_cast<int>(blockIdx.x) * 4 + wave) * 16, i0 = static_cast<int>(blockIdx.y) * 16;
  if (j0 >= p.n) return;
  const int8_t* wr = p.w + min(j0 + l16, p.n - 1) * p.w_stride + 16 * g;
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
  // register e: feature j0 + 4g + e of token i0 + l16
  const int i = i0 + l16;
  if (i >= p.m) return;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j0 + 4 * g + e < p.n) store_scaled<T>(p, i, j0 + 4 * g + e, acc[e]);
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
  const dim3 grid((ops->n + 63) / 64, (ops->m + 15) / 16);
  if (grid.y > 65535) return LRA_ERR_UNSUPPORTED;
  if (dtype == LRA_BF16) hipLaunchKernelGGL((matmul_i8_kernel<bf16_t>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((matmul_i8_kernel<float>), grid, dim3(256), 0, s, p);
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
