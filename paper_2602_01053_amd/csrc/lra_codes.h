// Caches of 8-bit codes (lra_attn8.h): kernel parameters, codes and their scales.
#pragma once

#include "lra_attn8.h"
#include "lra_batch.h"
#include "lra_prefill_util.h"

namespace lra {

// k_base, v_base: codes; kv_block_stride, kv_head_stride: bytes
struct Batch8Params : BatchParams {
  const uint8_t *k_scale, *v_scale;
  int64_t scale_block_stride;
  int32_t code;
  int32_t longest_first;            // tiles kernel: q tiles in the order of what they see
  int32_t head_shares;              // key shares of a kv head over all sequences, formed by their lengths (0: n_splits of every sequence or q tile)
  int32_t share_least;              // rows kernels: tiles of the shortest of those
};

// Block b of sequence t.
__device__ __forceinline__ int block8(const int32_t* table, int max_blocks_per_seq, int t, int b) {
  return table ? table[static_cast<int64_t>(t) * max_blocks_per_seq + b] : b;
}

// 2^(s - 127); 255 is not a number, 0 the denormal 2^-127: the exponent field, and the upper mantissa bit for those two.  (Without a
// branch: behind one, every load of a scale was waited for by itself.)
__device__ __forceinline__ float scale8(int s) {
  const uint32_t u = static_cast<uint32_t>(s);
  return __uint_as_float(u << 23 | (((u + 1u) & 255u) < 2u ? 0x00400000u : 0u));
}

// Exponent byte of the least power of two (2^-126 at least) that brings a value with these bits (sign cleared) to 448 = 1.75 x 2^8
// or 127 = 1.984375 x 2^6 at most: one more than the value's own exponent less 8 or 6 where its mantissa is larger than theirs.
template <int CODE>
__device__ __forceinline__ int least_scale8(uint32_t bits) {
  if (bits >= 0x7f800000u) return 255;
  const int e = CODE == LRA_E4M3 ? static_cast<int>((bits + 0x1fffffu) >> 23) - 8 : static_cast<int>((bits + 0x01ffffu) >> 23) - 6;
  return max(e, 1);
}

// What a wave's lanes have written to LDS, its other lanes read behind this (in order anyhow: for the compiler).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Codes that the launch reads once, past the caches' replacement: 64 k tokens of 8 kv heads take 31 us so instead of 36 (14 rows over a
// batch of 780 MB 4 % less); what the memory-side cache still holds comes a little later, 32 k tokens in 21.8 instead of 20.8 us.
__device__ __forceinline__ uint4 load_once(const uint8_t* src) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const pf_u32x4*>(src)));
}

// Sixteen bits as byte masks, four to a word.
__device__ __forceinline__ uint4 byte_masks(uint32_t bits) {
  auto word = [&](int c) __attribute__((always_inline)) -> uint32_t { return (((bits >> (4 * c)) & 15u) * 0x00204081u & 0x01010101u) * 255u; };
  return make_uint4(word(0), word(1), word(2), word(3));
}
// ... of the sixteen tokens from j0 on: ones for those below n and outside [cut_lo, cut_hi).
__device__ __forceinline__ uint4 token_masks(int j0, int n, int cut_lo, int cut_hi) {
  auto below = [](int k) __attribute__((always_inline)) -> uint32_t { return (1u << min(max(k, 0), 16)) - 1u; };
  return byte_masks(below(n - j0) & ~(below(cut_hi - j0) & ~below(cut_lo - j0)));
}

// The four codes of a word as floats.
template <int CODE>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (CODE == LRA_E4M3) {
    const pf_f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = static_cast<float>(static_cast<signed char>(w >> (8 * i)));
  }
}

// Four scaled values (at most 448 or 127 in magnitude) rounded to codes, to nearest, ties to even.
template <int CODE>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4]) {
  if constexpr (CODE == LRA_E4M3) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true));
  } else {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= (static_cast<uint32_t>(static_cast<int>(rintf(x[i]))) & 255u) << (8 * i);
    return r;
  }
}

hipError_t launch_attn8_rows_e4m3(const Batch8Params& p, int row_tiles, hipStream_t s);
hipError_t launch_attn8_rows_int8(const Batch8Params& p, int row_tiles, hipStream_t s);
// part_ml NULL: no states, the outputs themselves (n_splits 1)
hipError_t launch_attn8_tiles_e4m3(const Batch8Params& p, hipStream_t s);
hipError_t launch_attn8_tiles_int8(const Batch8Params& p, hipStream_t s);

}  // namespace lra
