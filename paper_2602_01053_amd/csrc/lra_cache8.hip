// The cache of 8-bit codes: new rows written into it, rows read back (declarations and contracts in lra_attn8.h).
#include "lra_attn8_plan.h"
#include "lra_codes.h"

namespace lra {

struct Append8Params {
  const void *k, *v, *l;  // new rows (l may be null)
  uint8_t *kc, *vc, *k_scale, *v_scale;
  void* lc;
  const int32_t *block_table, *seq_lens, *seq_start, *positions;
  int64_t k_token_stride, v_token_stride, l_token_stride, kv_block_stride, kv_head_stride, scale_block_stride, l_row_stride;
  int64_t items;
  int32_t n_kv_heads, rank, n_seqs, max_seq_len, max_blocks_per_seq, num_blocks, n_new, blocks_per_seq;
  float rope_theta;
};

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), off, kWave)));
  return v;
}

// Sine and cosine of 2 pi x turns, |turns| <= 1/2, from their power series about the nearest quarter turn, to 1e-12: rounded to fp32
// they are those of the exact angle but for one in 10^5, so that a key's codes do not depend on how its angle was reduced.  (The
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
// prompts and by its one chain (lengths, block id, rows, largest value, store) for a decode step.
template <typename T, int D, int CODE>
__global__ __launch_bounds__(256) void cache8_append_kernel(Append8Params p) {
  constexpr int H = D / 2, PP = D / 8, DV = D / 64;
  __shared__ float2 turn[16][H];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pairs = (p.n_kv_heads + 1) / 2;
  for (int64_t item = blockIdx.x; item < p.items; item += gridDim.x) {
    const int pair = static_cast<int>(item % pairs);
    const int64_t rest = item / pairs;
    const int t = static_cast<int>(rest / p.blocks_per_seq), bi = static_cast<int>(rest - static_cast<int64_t>(t) * p.blocks_per_seq);
    const int n = p.seq_lens[t];
    const int c0 = t > 0 ? min(max(p.seq_start[t], 0), p.n_new) : 0;
    const int c1 = t + 1 < p.n_seqs ? min(max(p.seq_start[t + 1], c0), p.n_new) : p.n_new;
    if (n > p.max_seq_len || c1 <= c0) continue;
    const int first = n - (c1 - c0);  // (negative: rows before the sequence)
    const int b = (max(first, 0) >> 4) + bi, j0 = b * 16;
    if (j0 >= n) continue;
    const int id = block8(p.block_table, p.max_blocks_per_seq, t, b);
    if (id < 0 || id >= p.num_blocks) continue;
    const int lo = max(first - j0, 0), hi = min(16, n - j0);  // slots [0, lo) are held already, [lo, hi) are new
    const int row0 = c0 + j0 - first;                          // row of slot 0
    if (p.rope_theta > 0.f) {
      const double rate = rope_rate_rev(tid % H, D, p.rope_theta);
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
        float x[PP], y[PP];
#pragma unroll
        for (int i = 0; i < PP; ++i) x[i] = y[i] = 0.f;
        uint32_t most = 0;
        if (fresh) {
          const T* src = static_cast<const T*>(p.k) + (row0 + s) * p.k_token_stride + static_cast<int64_t>(h) * D + part;
          load_values<T, PP>(src, x);
          load_values<T, PP>(src + H, y);
#pragma unroll
          for (int i = 0; i < PP; ++i) {
            if (p.rope_theta > 0.f) {
              const float2 cs = turn[s][part + i];
              const float a = x[i], c = y[i];
              // (each product rounded, as the definition has it, and not one of the two fused into the difference)
              x[i] = __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(c, cs.y));
              y[i] = __fadd_rn(__fmul_rn(c, cs.x), __fmul_rn(a, cs.y));
            }
            most = max(most, max(__float_as_uint(x[i]) & 0x7fffffffu, __float_as_uint(y[i]) & 0x7fffffffu));
          }
        }
        uint8_t* dst = p.kc + off + s * D + part;
        const int had = lo > 0 ? p.k_scale[soff] : 0;
        const int e = block_scale<CODE>(most, lo > 0, had);
        uint32_t cx[PP / 4], cy[PP / 4];
        const bool anew = s < lo && e != had;
        if (anew) {
#pragma unroll
          for (int i = 0; i < PP / 4; ++i) {
            float u[4], w[4];
            decode4<CODE>(reinterpret_cast<const uint32_t*>(dst)[i], u);
            decode4<CODE>(reinterpret_cast<const uint32_t*>(dst + H)[i], w);
#pragma unroll
            for (int c = 0; c < 4; ++c) x[4 * i + c] = ldexpf(u[c], had - e), y[4 * i + c] = ldexpf(w[c], had - e);
          }
        } else {
#pragma unroll
          for (int i = 0; i < PP; ++i) x[i] = ldexpf(x[i], 127 - e), y[i] = ldexpf(y[i], 127 - e);
        }
#pragma unroll
        for (int i = 0; i < PP / 4; ++i) {
          const float u[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]}, w[4] = {y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]};
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
        float x[16][DV];
        uint32_t most = 0;
#pragma unroll
        for (int s = 0; s < 16; ++s) {
#pragma unroll
          for (int c = 0; c < DV; ++c) x[s][c] = 0.f;
          if (s >= lo && s < hi) load_values<T, DV>(src + s * p.v_token_stride, x[s]);
#pragma unroll
          for (int c = 0; c < DV; ++c) most = max(most, __float_as_uint(x[s][c]) & 0x7fffffffu);
        }
        const int had = lo > 0 ? p.v_scale[soff] : 0;
        const int e = block_scale<CODE>(most, lo > 0, had);
#pragma unroll
        for (int c = 0; c < DV; ++c) {
          uint4* dst = reinterpret_cast<uint4*>(p.vc + off + (lane * DV + c) * 16);
          uint32_t was[4] = {0u, 0u, 0u, 0u};
          if (lo > 0 || hi < 16) {
            const uint4 w = *dst;
            was[0] = w.x, was[1] = w.y, was[2] = w.z, was[3] = w.w;
          }
          uint32_t out[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float u[4], z[4];
            decode4<CODE>(was[i], u);
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] = 4 * i + q < lo ? ldexpf(u[q], had - e) : ldexpf(x[4 * i + q][c], 127 - e);
            const uint32_t now = encode4<CODE>(z);
            // bytes from the first that changes to hi (earlier tokens keep their codes where the scale stays)
            const int f = min(max((e != had ? 0 : lo) - 4 * i, 0), 4), g = min(max(hi - 4 * i, 0), 4);
            const uint32_t mask = g <= f ? 0u : (g == 4 ? 0xffffffffu : (1u << (8 * g)) - 1u) & (f == 0 ? 0xffffffffu : f == 4 ? 0u : ~((1u << (8 * f)) - 1u));
            out[i] = (now & mask) | (was[i] & ~mask);
          }
          *dst = make_uint4(out[0], out[1], out[2], out[3]);
        }
        if (lane == 0) p.v_scale[soff] = static_cast<uint8_t>(e);
      }
    }
    if (pair == 0 && p.l != nullptr) {
      const int r = p.rank, cnt = (hi - lo) * r;
      for (int i = tid; i < cnt; i += 256) {
        const int s = lo + i / r, c = i - i / r * r;
        static_cast<T*>(p.lc)[(static_cast<int64_t>(id) * 16 + s) * p.l_row_stride + c] = static_cast<const T*>(p.l)[(row0 + s) * p.l_token_stride + c];
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
  int64_t items;
  int32_t units;  // of sixteen rows, per sequence
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
// before a wave as in cache8_append_kernel.
template <typename T, int D, int CODE>
__global__ __launch_bounds__(256) void cache8_gather_kernel(Gather8Params p) {
  constexpr int PK = D / 4, DV = D / 64;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int Hkv = p.dst.n_kv_heads, pairs = (Hkv + 1) / 2;
  for (int64_t item = blockIdx.x; item < p.items; item += gridDim.x) {
    const int pair = static_cast<int>(item % pairs);
    const int64_t rest = item / pairs;
    const int t = static_cast<int>(rest / p.units), i0 = 16 * static_cast<int>(rest - static_cast<int64_t>(t) * p.units);
    const int m = min(p.dst.seq_lens[t], p.dst.max_seq_len), n = min(p.seq_lens[t], p.max_seq_len);
    if (i0 >= m) continue;
    // row s of the sixteen: its source token, negative where there is none, and the block of that
    const int row = i0 + (lane & 15);
    int tok = row < m ? (p.kept ? p.kept[static_cast<int64_t>(t) * p.kept_stride + row] : row + n - p.dst.seq_lens[t]) : -1;
    if (tok >= n) tok = -1;
    int id = 0;
    if (tok >= 0) {
      id = block8(p.block_table, p.max_blocks_per_seq, t, tok >> 4);
      if (id < 0 || id >= p.num_blocks) tok = -1;
    }
    const int h = 2 * pair + (wave & 1);
    if (h < Hkv) {
      const int64_t hoff = static_cast<int64_t>(h) * p.kv_head_stride;
      if (wave < 2) {
        const int s = lane >> 2, part = (lane & 3) * PK;
        const int j = __shfl(tok, s, kWave), blk = __shfl(id, s, kWave);
        if (j >= 0) {
          const uint4* src = reinterpret_cast<const uint4*>(p.kc + blk * p.kv_block_stride + hoff + (j & 15) * D + part);
          const float sc = scale8(p.k_scale[blk * p.scale_block_stride + h]);
          T* dst = static_cast<T*>(const_cast<void*>(p.dst.k_base)) + kv_offset(p.dst, t, i0 + s, h) + part;
#pragma unroll
          for (int i = 0; i < PK / 16; ++i) {
            const uint4 v = src[i];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
#pragma unroll
        for (int s = 0; s < 16; ++s) {
          const int j = __builtin_amdgcn_readlane(tok, s), blk = __builtin_amdgcn_readlane(id, s);
          if (j < 0) continue;
          const uint8_t* src = p.vc + blk * p.kv_block_stride + hoff + lane * DV * 16 + (j & 15);
          const float sc = scale8(p.v_scale[blk * p.scale_block_stride + h]);
          float x[DV];
#pragma unroll
          for (int c = 0; c < DV; ++c) {
            float u[4];
            decode4<CODE>(src[c * 16], u);
            x[c] = u[0] * sc;
          }
          store_values<T, DV>(static_cast<T*>(const_cast<void*>(p.dst.v_base)) + kv_offset(p.dst, t, i0 + s, h) + lane * DV, x);
        }
      }
    }
    if (pair == 0) {
      const int r = p.dst.rank;
      for (int i = tid; i < 16 * 64; i += 256) {
        const int s = i >> 6, c = i & 63;
        const int j = __shfl(tok, s, kWave), blk = __shfl(id, s, kWave);
        if (j < 0 || c >= r) continue;
        static_cast<T*>(const_cast<void*>(p.dst.l))[l_offset(p.dst, t, i0 + s, 0) + c] =
            static_cast<const T*>(p.lc)[(static_cast<int64_t>(blk) * 16 + (j & 15)) * p.l_row_stride + c];
      }
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

constexpr int64_t kMostWorkgroups = 1 << 20;  // (further items in turns)

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
  p.rope_theta = rows->rope_theta;
  // c tokens touch (c + 30) / 16 blocks at most
  const int most = rows->max_new_per_seq < cache->max_seq_len ? rows->max_new_per_seq : cache->max_seq_len;
  p.blocks_per_seq = static_cast<int32_t>((static_cast<int64_t>(most) + 30) / 16);
  p.items = static_cast<int64_t>(cache->n_seqs) * p.blocks_per_seq * ((shape->n_kv_heads + 1) / 2);
  const dim3 grid(static_cast<unsigned>(p.items < kMostWorkgroups ? p.items : kMostWorkgroups));
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
  p.units = static_cast<int32_t>((static_cast<int64_t>(dst->max_seq_len) + 15) / 16);
  p.items = static_cast<int64_t>(dst->n_seqs) * p.units * ((shape->n_kv_heads + 1) / 2);
  const dim3 grid(static_cast<unsigned>(p.items < kMostWorkgroups ? p.items : kMostWorkgroups));
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_type(shape, src->code, [&](auto t_c, auto d_c, auto code_c) {
    hipLaunchKernelGGL((cache8_gather_kernel<decltype(t_c), decltype(d_c)::value, decltype(code_c)::value>), grid, dim3(256), 0, s, p);
  });
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
