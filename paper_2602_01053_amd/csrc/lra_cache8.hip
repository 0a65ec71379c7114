// The cache of 8-bit codes: new rows written into it, rows read back (declarations and contracts in lra_attn8.h).
#include <cmath>

#include "lra_attn8_plan.h"
#include "lra_codes.h"

namespace lra {

struct Append8Params {
  const void *k, *v, *l;  // new rows (l may be null)
  uint8_t *kc, *vc, *k_scale, *v_scale;
  void* lc;
  const int32_t *block_table, *seq_lens, *seq_start, *positions;
  int64_t k_token_stride, v_token_stride, l_token_stride, kv_block_stride, kv_head_stride, scale_block_stride, l_row_stride;
  uint32_t places;  // (block with new tokens, pair of kv heads) of a sequence
  int32_t n_kv_heads, rank, n_seqs, max_seq_len, max_blocks_per_seq, num_blocks, n_new;
  int32_t rotate;
  double first_rate, rate_powers[6];  // turns per position of pair 0; theta^(-2^(i+1) / d), i < 6
};

// Turns per position of pair i < 64: theta^(-2i / d) / 2 pi, from the powers that i's bits select.  (Left to the device's exp2 and log2
// in double precision, the rates took longer than the angles.)
__device__ __forceinline__ double rate_of(const Append8Params& p, int i) {
  double r = p.first_rate;
#pragma unroll
  for (int b = 0; b < 6; ++b) r *= i >> b & 1 ? p.rate_powers[b] : 1.0;
  return r;
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), off, kWave)));
  return v;
}

// Sine and cosine of 2 pi x turns, |turns| <= 1/2, from their power series about the nearest quarter turn, to 7e-12 (the sine's
// first missing term, at an eighth of a turn): rounded to fp32 they are those of the exact angle but for one in 10^5, so that a key's codes do not depend on how its angle was reduced.  (The
// hardware's v_sin_f32 is off by up to 1e-6, which moves one in 10^4 codes to the next.)
__device__ __forceinline__ void sincos_turns(double turns, float& sn, float& cs) {
  const double q = rint(4.0 * turns);
  const double a = (turns - 0.25 * q) * 6.283185307179586477, z = a * a;  // |a| <= pi / 4
  double s = -1.0 / 39916800.0, c = 1.0 / 479001600.0;
  s = fma(s, z, 1.0 / 362880.0), c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, -1.0 / 5040.0), c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, 1.0 / 120.0), c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, -1.0 / 6.0), c = fma(c, z, 1.0 / 24.0);
  s = fma(s * z, a, a), c = fma(fma(c, z, -0.5), z, 1.0);
  const int k = static_cast<int>(q) & 3;
  const float fs = static_cast<float>(s), fc = static_cast<float>(c);
  const float u = k & 1 ? fc : fs, w = k & 1 ? fs : fc;
  sn = k & 2 ? -u : u;
  cs = k == 1 || k == 2 ? -w : w;
}

template <typename T, int N>
__device__ __forceinline__ void load_values(const T* src, float (&x)[N]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (N >= 4) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const float4 v = reinterpret_cast<const float4*>(src)[i];
        x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
      }
    } else if constexpr (N == 2) {
      const float2 v = *reinterpret_cast<const float2*>(src);
      x[0] = v.x, x[1] = v.y;
    } else {
      x[0] = *src;
    }
  } else {
    if constexpr (N >= 8) {
#pragma unroll
      for (int i = 0; i < N / 8; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(src)[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[8 * i + 2 * e] = __uint_as_float(w[e] << 16), x[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    } else if constexpr (N == 2) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(src);
      x[0] = __uint_as_float(w << 16), x[1] = __uint_as_float(w & 0xffff0000u);
    } else {
      x[0] = bf16_to_f32(*src);
    }
  }
}

// A wave's block of one kv head: scale from the largest new value and, with earlier tokens, the one it had.
template <int CODE>
__device__ __forceinline__ int block_scale(uint32_t most_bits, bool has_old, int had) {
  const int e = least_scale8<CODE>(wave_max_u32(most_bits));
  return has_old ? max(e, had) : e;
}

// One workgroup of four waves per (sequence, block with new tokens, pair of kv heads): keys and values of the two heads.  The
// keys of a block lie before a wave as 16 tokens x 4 parts of a row and its rotation partner, the values as one or two
// dimensions a lane, all sixteen tokens each: what a lane stores is 16 bytes in a row, and the largest value is 32 values a
// lane and one reduction away.  Angles are formed once for both heads and handed round in LDS.  Bound by memory for long
// prompts (four of up to 4096 tokens, 51 MB: 13 to 15 us, 3.4 to 3.8 TB/s) and by its one chain (lengths, block id, rows, largest value,
// store) for a decode step (64 sequences: 5.3 us).
template <typename T, int D, int CODE>
__global__ __launch_bounds__(256) void cache8_append_kernel(Append8Params p) {
  constexpr int H = D / 2, PP = D / 8, DV = D / 64;
  __shared__ float2 turn[16][H];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t pairs = static_cast<uint32_t>(p.n_kv_heads + 1) / 2;
  const double rate = p.rotate ? rate_of(p, tid % H) : 0.0;
  for (int t = blockIdx.y; t < p.n_seqs; t += gridDim.y)
  for (uint32_t place = blockIdx.x; place < p.places; place += gridDim.x) {
    const int bi = static_cast<int>(place / pairs), pair = static_cast<int>(place - static_cast<uint32_t>(bi) * pairs);
    // (three requests, one round trip)
    const int n = p.seq_lens[t], at = p.seq_start[t], end = p.seq_start[t + 1];
    const int c0 = t > 0 ? min(max(at, 0), p.n_new) : 0;
    const int c1 = t + 1 < p.n_seqs ? min(max(end, c0), p.n_new) : p.n_new;
    if (n > p.max_seq_len || c1 <= c0) continue;
    const int first = n - (c1 - c0);  // (negative: rows before the sequence)
    const int b = (max(first, 0) >> 4) + bi, j0 = b * 16;
    if (j0 >= n) continue;
    const int id = block8(p.block_table, p.max_blocks_per_seq, t, b);
    if (id < 0 || id >= p.num_blocks) continue;
    const int lo = max(first - j0, 0), hi = min(16, n - j0);  // slots [0, lo) are held already, [lo, hi) are new
    const int row0 = c0 + j0 - first;                          // row of slot 0
    if (p.rotate) {
      for (int s = tid / H; s < hi; s += 256 / H)
        if (s >= lo) {
          const int pos = p.positions ? p.positions[row0 + s] : j0 + s;
          const double rev = static_cast<double>(pos) * rate;
          float sn, cs;
          sincos_turns(rev - rint(rev), sn, cs);
          turn[s][tid % H] = make_float2(cs, sn);
        }
      __syncthreads();
    }
    const int h = 2 * pair + (wave & 1);
    if (h < p.n_kv_heads) {
      const int64_t off = static_cast<int64_t>(id) * p.kv_block_stride + static_cast<int64_t>(h) * p.kv_head_stride;
      const int64_t soff = static_cast<int64_t>(id) * p.scale_block_stride + h;
      if (wave < 2) {
        const int s = lane >> 2, part = (lane & 3) * PP;
        const bool fresh = s >= lo && s < hi;
        // (slots that get no row: the nearest that does, zeroed; everything is requested before anything is waited for)
        const T* src = static_cast<const T*>(p.k) + (row0 + min(max(s, lo), hi - 1)) * p.k_token_stride + static_cast<int64_t>(h) * D + part;
        uint8_t* const dst = p.kc + off + s * D + part;
        float x[PP], y[PP];
        load_values<T, PP>(src, x);
        load_values<T, PP>(src + H, y);
        uint32_t wx[PP / 4], wy[PP / 4];  // codes of earlier tokens
        int had = 0;
        if (lo > 0) {
          had = p.k_scale[soff];
#pragma unroll
          for (int i = 0; i < PP / 4; ++i) wx[i] = reinterpret_cast<const uint32_t*>(dst)[i], wy[i] = reinterpret_cast<const uint32_t*>(dst + H)[i];
        }
        if (p.rotate) {
#pragma unroll
          for (int i = 0; i < PP; ++i) {
            const float2 cs = turn[s][part + i];  // (of slots that get no row: anything)
            const float a = x[i], c = y[i];
            // (each product rounded, as the definition has it, and not one of the two fused into the difference)
            x[i] = __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(c, cs.y));
            y[i] = __fadd_rn(__fmul_rn(c, cs.x), __fmul_rn(a, cs.y));
          }
        }
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < PP; ++i) most = max(most, max(__float_as_uint(x[i]) & 0x7fffffffu, __float_as_uint(y[i]) & 0x7fffffffu));
        const int e = block_scale<CODE>(fresh ? most : 0u, lo > 0, had);
        const bool anew = s < lo && e != had;
        int by = 127 - e;
        if (lo > 0) {  // (uniform)
          if (s < lo) by = had - e;
#pragma unroll
          for (int i = 0; i < PP / 4; ++i) {
            float u[4], w[4];
            decode4<CODE>(wx[i], u);
            decode4<CODE>(wy[i], w);
#pragma unroll
            for (int c = 0; c < 4; ++c) x[4 * i + c] = s < lo ? u[c] : x[4 * i + c], y[4 * i + c] = s < lo ? w[c] : y[4 * i + c];
          }
        }
        uint32_t cx[PP / 4], cy[PP / 4];
#pragma unroll
        for (int i = 0; i < PP / 4; ++i) {
          float u[4], w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) u[c] = ldexpf(x[4 * i + c], by), w[c] = ldexpf(y[4 * i + c], by);
          cx[i] = encode4<CODE>(u), cy[i] = encode4<CODE>(w);
        }
        if (fresh || anew) {
          if constexpr (PP == 16) {
            *reinterpret_cast<uint4*>(dst) = make_uint4(cx[0], cx[1], cx[2], cx[3]);
            *reinterpret_cast<uint4*>(dst + H) = make_uint4(cy[0], cy[1], cy[2], cy[3]);
          } else {
            *reinterpret_cast<uint2*>(dst) = make_uint2(cx[0], cx[1]);
            *reinterpret_cast<uint2*>(dst + H) = make_uint2(cy[0], cy[1]);
          }
        }
        if (lane == 0) p.k_scale[soff] = static_cast<uint8_t>(e);
      } else {
        const T* src = static_cast<const T*>(p.v) + row0 * p.v_token_stride + static_cast<int64_t>(h) * D + lane * DV;
        uint4* const dst = reinterpret_cast<uint4*>(p.vc + off + lane * DV * 16);
        float x[16][DV];
#pragma unroll
        for (int s = 0; s < 16; ++s) load_values<T, DV>(src + min(max(s, lo), hi - 1) * p.v_token_stride, x[s]);
        uint4 was[DV];
        int had = 0;
        if (lo > 0 || hi < 16) {
          if (lo > 0) had = p.v_scale[soff];
#pragma unroll
          for (int c = 0; c < DV; ++c) was[c] = dst[c];
        } else {
#pragma unroll
          for (int c = 0; c < DV; ++c) was[c] = make_uint4(0u, 0u, 0u, 0u);
        }
        uint32_t most = 0;  // (rows requested twice count once)
#pragma unroll
        for (int s = 0; s < 16; ++s)
#pragma unroll
          for (int c = 0; c < DV; ++c) most = max(most, __float_as_uint(x[s][c]) & 0x7fffffffu);
        const int e = block_scale<CODE>(most, lo > 0, had);
        // bytes from the first that changes to hi (earlier tokens keep their codes where the scale stays)
        const uint4 mask = byte_masks(((1u << hi) - 1u) & ~((1u << (e != had ? 0 : lo)) - 1u));
        const uint32_t ms[4] = {mask.x, mask.y, mask.z, mask.w};
#pragma unroll
        for (int c = 0; c < DV; ++c) {
          const uint32_t old[4] = {was[c].x, was[c].y, was[c].z, was[c].w};
          uint32_t out[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float z[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] = ldexpf(x[4 * i + q][c], 127 - e);
            if (lo > 4 * i) {  // (uniform)
              float u[4];
              decode4<CODE>(old[i], u);
#pragma unroll
              for (int q = 0; q < 4; ++q) z[q] = 4 * i + q < lo ? ldexpf(u[q], had - e) : z[q];
            }
            out[i] = (encode4<CODE>(z) & ms[i]) | (old[i] & ~ms[i]);
          }
          dst[c] = make_uint4(out[0], out[1], out[2], out[3]);
        }
        if (lane == 0) p.v_scale[soff] = static_cast<uint8_t>(e);
      }
    }
    if (pair == 0 && p.l != nullptr) {
      const int c = min(lane, p.rank - 1);
      T x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = static_cast<const T*>(p.l)[(row0 + min(max(4 * i + wave, lo), hi - 1)) * p.l_token_stride + c];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = 4 * i + wave;
        if (s >= lo && s < hi && lane < p.rank) static_cast<T*>(p.lc)[(static_cast<int64_t>(id) * 16 + s) * p.l_row_stride + c] = x[i];
      }
    }
    __syncthreads();  // (the angles of the next item)
  }
}

struct Gather8Params {
  const uint8_t *kc, *vc, *k_scale, *v_scale;
  const void* lc;
  const int32_t *block_table, *seq_lens, *kept;
  int64_t kv_block_stride, kv_head_stride, scale_block_stride, l_row_stride, kept_stride;
  int32_t max_blocks_per_seq, num_blocks, max_seq_len;
  Params dst;  // k_base, v_base, l and their layout, seq_lens, max_seq_len, n_kv_heads, rank
  uint32_t places;  // (sixteen rows, pair of kv heads) of a sequence
  int32_t n_seqs;
};

template <typename T, int N>
__device__ __forceinline__ void store_values(T* dst, const float (&x)[N]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; ++i) dst[i] = x[i];
  } else {
    // (products of a code and a power of two: exact, but for NaN)
    if constexpr (N == 1) {
      *dst = f32_to_bf16(x[0]);
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) reinterpret_cast<uint32_t*>(dst)[i] = pf_pack2(x[2 * i], x[2 * i + 1]);
    }
  }
}

// One workgroup of four waves per (sequence, sixteen rows of dst, pair of kv heads): keys and values of the two heads, laid out
// before a wave as in cache8_append_kernel.  4096 kept of 16384 rows take 11.3 to 12.6 us (25 MB needed; a kept token's 16 bytes of V a
// dimension are one byte's worth), 64 sequences' last blocks 6: a chain (lengths, kept row, block id, codes, store).
template <typename T, int D, int CODE>
__global__ __launch_bounds__(256) void cache8_gather_kernel(Gather8Params p) {
  constexpr int PK = D / 4, DV = D / 64;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int Hkv = p.dst.n_kv_heads;
  const uint32_t pairs = static_cast<uint32_t>(Hkv + 1) / 2;
  for (int t = blockIdx.y; t < p.n_seqs; t += gridDim.y)
  for (uint32_t place = blockIdx.x; place < p.places; place += gridDim.x) {
    const uint32_t unit = place / pairs;
    const int pair = static_cast<int>(place - unit * pairs), i0 = static_cast<int>(unit) * 16;
    const int m_all = p.dst.seq_lens[t], n_all = p.seq_lens[t];
    const int m = min(m_all, p.dst.max_seq_len), n = min(n_all, p.max_seq_len);
    if (i0 >= m) continue;
    // (entries of dst's table behind its last block are not read: asked for beside the lengths, the entry came 0.15 us sooner)
    const int dst_id = p.dst.block_size == 0 ? 0 : p.dst.block_table[static_cast<int64_t>(t) * p.dst.max_blocks_per_seq + static_cast<int>(unit)];
    // (the sixteen rows lie in one block of dst; looked up row by row, behind the stores, the ids took most of the kernel's time)
    const int64_t dst_block = dst_id;
    const int64_t kv_base = p.dst.block_size == 0 ? i0 * p.dst.kv_token_stride : dst_block * p.dst.kv_block_stride;
    const int64_t l_base = (p.dst.block_size == 0 ? i0 : dst_block * 16) * p.dst.l_row_stride;
    // row s of the sixteen: its source token, negative where there is none, and the block of that
    const int row = i0 + (lane & 15);
    int tok = row < m ? (p.kept ? p.kept[static_cast<int64_t>(t) * p.kept_stride + row] : row + n - m_all) : -1;
    if (tok >= n) tok = -1;
    int id = 0;
    if (tok >= 0) {
      id = block8(p.block_table, p.max_blocks_per_seq, t, tok >> 4);
      if (id < 0 || id >= p.num_blocks) tok = -1, id = 0;
    }
    const int h = 2 * pair + (wave & 1);
    if (h < Hkv) {
      // (the scale of this lane's row: one request for the sixteen)
      const int scale_byte = (wave < 2 ? p.k_scale : p.v_scale)[id * p.scale_block_stride + h];
      const int64_t hoff = static_cast<int64_t>(h) * p.kv_head_stride;
      if (wave < 2) {
        const int s = lane >> 2, part = (lane & 3) * PK;
        const int j = __shfl(tok, s, kWave), blk = __shfl(id, s, kWave);  // (a row without a source: block 0, of which nothing is stored)
        const uint4* src = reinterpret_cast<const uint4*>(p.kc + blk * p.kv_block_stride + hoff + (j & 15) * D + part);
        uint4 v[PK / 16];
#pragma unroll
        for (int i = 0; i < PK / 16; ++i) v[i] = src[i];
        const float sc = scale8(__shfl(scale_byte, s, kWave));
        T* dst = static_cast<T*>(const_cast<void*>(p.dst.k_base)) + kv_base + s * p.dst.kv_token_stride + h * p.dst.kv_head_stride + part;
        if (j >= 0) {
#pragma unroll
          for (int i = 0; i < PK / 16; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            float x[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float u[4];
              decode4<CODE>(w[q], u);
#pragma unroll
              for (int c = 0; c < 4; ++c) x[4 * q + c] = u[c] * sc;
            }
            store_values<T, 16>(dst + 16 * i, x);
          }
        }
      } else {
        // sixteen tokens of a lane's dimensions for every row (rows of one block: from the cache near the unit), of which one byte
        // counts; eight rows at a time
        T* const dst = static_cast<T*>(const_cast<void*>(p.dst.v_base)) + kv_base + h * p.dst.kv_head_stride + lane * DV;
#pragma unroll 1
        for (int s0 = 0; s0 < 16; s0 += 8) {
          uint4 v[8][DV];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int blk = __builtin_amdgcn_readlane(id, s0 + q);
            const uint4* src = reinterpret_cast<const uint4*>(p.vc + blk * p.kv_block_stride + hoff) + lane * DV;
#pragma unroll
            for (int c = 0; c < DV; ++c) v[q][c] = src[c];
          }
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int j = __builtin_amdgcn_readlane(tok, s0 + q);
            if (j < 0) continue;
            const float sc = scale8(__builtin_amdgcn_readlane(scale_byte, s0 + q));
            float x[DV];
#pragma unroll
            for (int c = 0; c < DV; ++c) {
              const uint32_t four = j & 8 ? (j & 4 ? v[q][c].w : v[q][c].z) : (j & 4 ? v[q][c].y : v[q][c].x);
              float u[4];
              decode4<CODE>(four >> (8 * (j & 3)), u);
              x[c] = u[0] * sc;
            }
            store_values<T, DV>(dst + (s0 + q) * p.dst.kv_token_stride, x);
          }
        }
      }
    }
    if (pair == 0) {
      const int r = p.dst.rank, c = min(lane, r - 1);
      T x[4];
      int js[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = 4 * i + wave, blk = __shfl(id, s, kWave);
        js[i] = __shfl(tok, s, kWave);
        x[i] = static_cast<const T*>(p.lc)[(static_cast<int64_t>(blk) * 16 + (js[i] & 15)) * p.l_row_stride + c];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (js[i] >= 0 && lane < r) static_cast<T*>(const_cast<void*>(p.dst.l))[l_base + (4 * i + wave) * p.dst.l_row_stride + c] = x[i];
    }
  }
}

template <typename F>
static void by_type(const lra_shape* sh, int code, F launch) {
  auto with_code = [&](auto t_c, auto d_c) {
    if (code == LRA_E4M3) launch(t_c, d_c, std::integral_constant<int, LRA_E4M3>{});
    else launch(t_c, d_c, std::integral_constant<int, LRA_INT8>{});
  };
  auto with_dim = [&](auto t_c) {
    if (sh->head_dim == 128) with_code(t_c, std::integral_constant<int, 128>{});
    else with_code(t_c, std::integral_constant<int, 64>{});
  };
  if (sh->dtype == LRA_BF16) with_dim(bf16_t{});
  else with_dim(float{});
}

// The grid of `units` by pairs of kv heads (x) and sequences (y), what is beyond its bounds in turns; false: too many for 32 bits.
static bool place_grid(int64_t units, int n_kv_heads, int n_seqs, uint32_t& places, dim3& grid) {
  const int64_t n = units * ((n_kv_heads + 1) / 2);
  if (n > (int64_t{1} << 31)) return false;
  places = static_cast<uint32_t>(n);
  grid = dim3(static_cast<unsigned>(n < (1 << 20) ? n : (1 << 20)), n_seqs < 4096 ? n_seqs : 4096);
  return true;
}

}  // namespace lra

using namespace lra;

extern "C" {

lra_status lra_cache8_append(const lra_shape* shape, const lra_cache8* cache, const lra_new_rows* rows, void* stream) {
  const lra_status st = check_new_rows(shape, cache, rows);
  if (st != LRA_OK) return st;
  Append8Params p{};
  p.k = rows->k;
  p.v = rows->v;
  p.l = rows->l;
  p.kc = static_cast<uint8_t*>(cache->k);
  p.vc = static_cast<uint8_t*>(cache->v);
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.lc = cache->l;
  p.block_table = cache->block_table;
  p.seq_lens = cache->seq_lens;
  p.seq_start = rows->seq_start;
  p.positions = rows->positions;
  p.k_token_stride = rows->k_token_stride;
  p.v_token_stride = rows->v_token_stride;
  p.l_token_stride = rows->l_token_stride;
  p.kv_block_stride = cache->kv_block_stride;
  p.kv_head_stride = cache->kv_head_stride;
  p.scale_block_stride = cache->scale_block_stride ? cache->scale_block_stride : shape->n_kv_heads;
  p.l_row_stride = cache->l_row_stride ? cache->l_row_stride : shape->rank;
  p.n_kv_heads = shape->n_kv_heads;
  p.rank = shape->rank;
  p.n_seqs = cache->n_seqs;
  p.max_seq_len = cache->max_seq_len;
  p.max_blocks_per_seq = cache->max_blocks_per_seq;
  p.num_blocks = cache->num_blocks;
  p.n_new = rows->n_new;
  p.rotate = rows->rope_theta > 0.f;
  if (p.rotate) {
    p.first_rate = 0.15915494309189533577;  // 1 / 2 pi
    for (int i = 0; i < 6; ++i) p.rate_powers[i] = std::pow(static_cast<double>(rows->rope_theta), -2.0 * (1 << i) / shape->head_dim);
  }
  // c tokens touch (c + 30) / 16 blocks at most
  const int most = rows->max_new_per_seq < cache->max_seq_len ? rows->max_new_per_seq : cache->max_seq_len;
  dim3 grid;
  if (!place_grid((static_cast<int64_t>(most) + 30) / 16, shape->n_kv_heads, cache->n_seqs, p.places, grid)) return LRA_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_type(shape, cache->code, [&](auto t_c, auto d_c, auto code_c) {
    hipLaunchKernelGGL((cache8_append_kernel<decltype(t_c), decltype(d_c)::value, decltype(code_c)::value>), grid, dim3(256), 0, s, p);
  });
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

lra_status lra_cache8_gather(const lra_shape* shape, const lra_cache8* src, const int32_t* kept, int64_t kept_stride,
                             const lra_cache* dst, void* stream) {
  lra_status st = check_cache8(shape, src);
  if (st != LRA_OK) return st;
  st = check_common(shape, dst);
  if (st != LRA_OK) return st;
  if (dst->n_seqs != src->n_seqs) return LRA_ERR_SHAPE;
  if (kept && kept_stride < dst->max_seq_len) return LRA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(kept) & 3) return LRA_ERR_SHAPE;
  // (a row's index is the position by which its adapter part is rotated)
  if (shape->key_rope_theta > 0.f && kept) return LRA_ERR_UNSUPPORTED;
  if (dst->k_base == src->k || dst->k_base == src->v || dst->v_base == src->k || dst->v_base == src->v || dst->l == src->l) return LRA_ERR_SHAPE;
  Gather8Params p{};
  p.kc = static_cast<const uint8_t*>(src->k);
  p.vc = static_cast<const uint8_t*>(src->v);
  p.k_scale = src->k_scale;
  p.v_scale = src->v_scale;
  p.lc = src->l;
  p.block_table = src->block_table;
  p.seq_lens = src->seq_lens;
  p.kept = kept;
  p.kept_stride = kept_stride;
  p.kv_block_stride = src->kv_block_stride;
  p.kv_head_stride = src->kv_head_stride;
  p.scale_block_stride = src->scale_block_stride ? src->scale_block_stride : shape->n_kv_heads;
  p.l_row_stride = src->l_row_stride ? src->l_row_stride : shape->rank;
  p.max_blocks_per_seq = src->max_blocks_per_seq;
  p.num_blocks = src->num_blocks;
  p.max_seq_len = src->max_seq_len;
  p.dst.k_base = dst->k_base;
  p.dst.v_base = dst->v_base;
  p.dst.l = dst->l;
  p.dst.block_table = dst->block_table;
  p.dst.seq_lens = dst->seq_lens;
  p.dst.max_seq_len = dst->max_seq_len;
  p.dst.kv_token_stride = dst->kv_token_stride;
  p.dst.kv_head_stride = dst->kv_head_stride;
  p.dst.kv_block_stride = dst->kv_block_stride;
  p.dst.block_size = dst->block_size;
  p.dst.max_blocks_per_seq = dst->max_blocks_per_seq;
  p.dst.l_row_stride = dst->l_row_stride ? dst->l_row_stride : shape->rank;
  p.dst.n_kv_heads = shape->n_kv_heads;
  p.dst.rank = shape->rank;
  p.n_seqs = dst->n_seqs;
  dim3 grid;
  if (!place_grid((static_cast<int64_t>(dst->max_seq_len) + 15) / 16, shape->n_kv_heads, dst->n_seqs, p.places, grid)) return LRA_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_type(shape, src->code, [&](auto t_c, auto d_c, auto code_c) {
    hipLaunchKernelGGL((cache8_gather_kernel<decltype(t_c), decltype(d_c)::value, decltype(code_c)::value>), grid, dim3(256), 0, s, p);
  });
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
