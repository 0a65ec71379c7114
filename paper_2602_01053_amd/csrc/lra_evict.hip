// Cutting caches to a budget of tokens: lra_evict_select and lra_cache_gather of the header.
#include "lra_attn.h"
#include "lra_common.h"
#include "lra_decode_util.h"
#include "lra_plan.h"

namespace lra {

struct SelectParams {
  const int32_t* seq_lens;
  const float* weights;
  int32_t* kept;
  int32_t* new_lens;
  int64_t weights_stride, kept_stride;
  int32_t max_seq_len, budget, sinks, recent;
};

// Bits that order as the weights do, NaN below everything, -0 as 0; zero stands for no weight at all.
__device__ __forceinline__ uint32_t order_bits(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  const uint32_t o = u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
  return w != w ? 1u : o;
}

// One workgroup of sixteen waves per sequence.  The weights between sinks and recent tokens are cut into sixteen runs, one
// per wave, lane l of a wave taking every 64th of its run: loads are whole lines, and the order of tokens is that of (wave,
// step, lane).  The k-th largest is found digit by digit, eight bits at a time, from a histogram of those that agree with it
// in all digits before; of weights less the smallest, from the highest bit that the largest has, since bits that all have
// would put every weight into one counter (weights of a long tail have few exponents, and half of them the smallest one), and
// with four counters per digit, side by side, for the lanes that count the same one.  Once 64 weights or fewer are left, a
// wave ranks them against each other (after two digits of 64 k weights, usually).  Then every wave counts what it keeps,
// sixteen counts are added up, and every wave writes its own.
// A pass over the weights is bound by the one compute unit: at 64 k weights loading takes 3 us, their range 3.5, the first
// digit 7, the second 3, the list of the last few 3, counting 2.4 and writing 7 of 34; at 16 k all 11.7.  (First digits of raw
// bits in sixteen counters each, one set per wave, 20 and 63 us; weights in fours, kept tokens and candidates through lists in
// LDS: level.)
// K > 0: the lane's K weights stay in registers (K * 1024 weights at most); K == 0: read again for every pass.
template <int K>
__global__ __launch_bounds__(1024) void evict_select_kernel(SelectParams p) {
  __shared__ __align__(16) uint32_t hist[256][4];
  __shared__ uint32_t range_s[2][16];
  __shared__ uint32_t pick_s[3];
  __shared__ uint32_t few_s[64], few_n;
  __shared__ int count_s[2][16];
  const int lane = threadIdx.x & 63, tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x;
  const int n = max(0, min(p.seq_lens[t], p.max_seq_len));
  int32_t* kept = p.kept + t * p.kept_stride;
  __syncthreads();  // (new_lens may be seq_lens)
  const int m = min(n, p.budget);
  if (tid == 0) p.new_lens[t] = m;
  if (n <= p.budget) {
    for (int i = tid; i < n; i += 1024) kept[i] = i;
    return;
  }
  const int cnt = n - p.sinks - p.recent;
  int want = m - p.sinks - p.recent;  // of the cnt weights between, fewer than there are
  const float* w = p.weights + t * p.weights_stride + p.sinks;
  const int steps = K > 0 ? K : (cnt + 1023) / 1024;
  const int first = wave * steps * 64 + lane;
  uint32_t held[K > 0 ? K : 1];
  uint32_t base = 0u;  // (K == 0: taken off what is read again)
  auto load = [&](int i) __attribute__((always_inline)) {
    const uint32_t u = order_bits(w[min(first + 64 * i, cnt - 1)]) - base;
    return first + 64 * i < cnt ? u : 0u;
  };
  if (want > 0) {
    if constexpr (K > 0) {
#pragma unroll
      for (int i = 0; i < K; ++i) held[i] = load(i);
    }
  }
  for (int i = tid; i < p.sinks; i += 1024) kept[i] = i;
  for (int i = tid; i < p.recent; i += 1024) kept[m - p.recent + i] = n - p.recent + i;
  if (want == 0) return;
  (&hist[0][0])[tid] = 0u;
  if (tid == 0) few_n = 0u;
  // f(bits) for the lane's weights (zero past the end)
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (K > 0) {
#pragma unroll
      for (int i = 0; i < K; ++i) {
        f(held[i]);
        if ((i & 7) == 7) __builtin_amdgcn_sched_barrier(0);  // (or the temporaries of all steps live at once)
      }
    } else {
      for (int i = 0; i < steps; ++i) f(load(i));
    }
  };

  uint32_t lo = 0xffffffffu, hi = 0u;
  each([&](uint32_t u) __attribute__((always_inline)) {
    lo = min(lo, u - 1u);
    hi = max(hi, u);
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    lo = min(lo, static_cast<uint32_t>(__shfl_xor(static_cast<int>(lo), off)));
    hi = max(hi, static_cast<uint32_t>(__shfl_xor(static_cast<int>(hi), off)));
  }
  if (lane == 0) {
    range_s[0][wave] = lo;
    range_s[1][wave] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo = min(lo, range_s[0][i]);
    hi = max(hi, range_s[1][i]);
  }
  // From here on weights are counted from below the smallest: 1 for that one, still 0 for what stands past the end.
  const uint32_t range = hi - lo;  // (lo is one less than the smallest)
  if constexpr (K > 0) {
#pragma unroll
    for (int i = 0; i < K; ++i) held[i] = held[i] == 0u ? 0u : held[i] - lo;
  }
  base = lo;
  // The threshold: weights with (u >> shift) > cut stay, and `want` of the `left` weights with (u >> shift) == cut.
  // (Zeros agree with a cut of zero only, and are then counted among the smallest: never wanted.)
  int shift = range == 1u ? 0 : 32 - __builtin_clz(range), left = cnt;
  uint32_t cut = range == 1u ? 1u : 0u;
  auto agrees = [&](uint32_t u) __attribute__((always_inline)) -> bool { return ((u >> (shift - 1)) >> 1) == cut; };  // (shift: 1 to 32)
  while (shift > 0 && left > 64) {
    const int width = min(8, shift);
    const int below = shift - width;
    const uint32_t mask = (1u << width) - 1u;
    each([&](uint32_t u) __attribute__((always_inline)) {
      if (agrees(u)) atomicAdd(&hist[(u >> below) & mask][lane & 3], 1u);
    });
    __syncthreads();
    if (wave == 0) {
      // lane l: digits 255 - 4 l .. 252 - 4 l, so that a sum over the lanes before runs from the largest digit
      uint32_t c[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint4* at = reinterpret_cast<uint4*>(&hist[255 - 4 * lane - k][0]);
        const uint4 four = *at;
        c[k] = (four.x + four.y) + (four.z + four.w);
        *at = make_uint4(0u, 0u, 0u, 0u);  // (for the next digit)
      }
      const uint32_t sum = (c[0] + c[1]) + (c[2] + c[3]);
      uint32_t before = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = static_cast<uint32_t>(__shfl_up(static_cast<int>(before), off));
        if (lane >= off) before += o;
      }
      before -= sum;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (before < static_cast<uint32_t>(want) && static_cast<uint32_t>(want) <= before + c[k]) {
          pick_s[0] = static_cast<uint32_t>(255 - 4 * lane - k);
          pick_s[1] = static_cast<uint32_t>(want) - before;
          pick_s[2] = c[k];
        }
        before += c[k];
      }
    }
    __syncthreads();  // (pick_s is written next behind the barrier of the next digit)
    cut = (shift == 32 ? 0u : cut << width) | pick_s[0];
    want = static_cast<int>(pick_s[1]);
    left = static_cast<int>(pick_s[2]);
    shift = below;
  }
  if (shift > 0) {
    // 64 weights or fewer: in any order to LDS, where every lane of every wave counts those above its own
    each([&](uint32_t u) __attribute__((always_inline)) {
      if (u != 0u && agrees(u)) few_s[atomicAdd(&few_n, 1u)] = u;
    });
    __syncthreads();
    left = static_cast<int>(few_n);
    const uint32_t mine = lane < left ? few_s[lane] : 0u;
    int above = 0, equal = 0;
    for (int i = 0; i < left; ++i) {
      const uint32_t o = few_s[i];
      above += o > mine;
      equal += o == mine;
    }
    const uint64_t is = __builtin_amdgcn_ballot_w64(lane < left && above < want && want <= above + equal);
    const int who = __builtin_ctzll(is);
    cut = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(mine), who));
    want -= __builtin_amdgcn_readlane(above, who);
    left = __builtin_amdgcn_readlane(equal, who);
  }
  // u > cut stays, and the first `want` of the `left` with u == cut
  cut = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(cut)));
  want = __builtin_amdgcn_readfirstlane(want);
  left = __builtin_amdgcn_readfirstlane(left);
  int above = 0, equal = 0;
  each([&](uint32_t u) __attribute__((always_inline)) {
    above += u > cut;
    equal += u == cut;
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    above += __shfl_xor(above, off);
    equal += __shfl_xor(equal, off);
  }
  if (lane == 0) {
    count_s[0][wave] = above;
    count_s[1][wave] = equal;
  }
  __syncthreads();
  int eq_before = 0, at = p.sinks;
  for (int v = 0; v < wave; ++v) {
    at += __builtin_amdgcn_readfirstlane(count_s[0][v]);
    eq_before += __builtin_amdgcn_readfirstlane(count_s[1][v]);
  }
  at += min(eq_before, want);
  asm volatile("" : "+s"(cut));  // (or the 2 K comparisons of the counts are kept, in scalar registers that there are not)
  const bool all_equal_stay = want >= left;
  // (K > 0, at most 64 k weights: lanes that keep nothing store outside the resource, without a branch a step)
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(kept + p.sinks, K > 0 ? static_cast<uint32_t>(m - p.sinks - p.recent) * 4u : 0u);
  auto below_me = [&](uint64_t mask) __attribute__((always_inline)) -> int {
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0u));
  };
  auto emit = [&](int i, uint32_t u) __attribute__((always_inline)) {  // (cut is a weight's, not zero)
    bool stay = u >= cut;
    if (!all_equal_stay) {
      const uint64_t eq = __builtin_amdgcn_ballot_w64(u == cut);
      stay = u > cut || (u == cut && eq_before + below_me(eq) < want);
      eq_before += __builtin_popcountll(eq);
    }
    const uint64_t all = __builtin_amdgcn_ballot_w64(stay);
    if constexpr (K > 0)
      __builtin_amdgcn_raw_buffer_store_b32(p.sinks + first + 64 * i, rs, stay ? (at - p.sinks + below_me(all)) * 4 : static_cast<int>(kOob), 0, 0);
    else if (stay)
      kept[at + below_me(all)] = p.sinks + first + 64 * i;
    at += __builtin_popcountll(all);
  };
  if constexpr (K > 0) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
      emit(i, held[i]);
      if ((i & 7) == 7) __builtin_amdgcn_sched_barrier(0);
    }
  } else {
    for (int i = 0; i < steps; ++i) emit(i, load(i));
  }
}

struct GatherSide {
  void* k;
  void* v;
  void* l;
  const int32_t* block_table;
  int64_t kv_token_stride, kv_head_stride, kv_block_stride, l_row_stride, l_adapter_stride;
  int32_t block_size, max_blocks_per_seq, max_seq_len;
};
struct GatherParams {
  GatherSide src, dst;
  const int32_t* kept;
  const int32_t* new_lens;
  const float* weights;
  float* dst_weights;
  int64_t kept_stride, weights_stride, dst_weights_stride;
  int32_t n_kv_heads, row_pieces;  // 16-byte pieces of a K or V row
  int32_t l_bytes, n_adapters;     // bytes of an L row
  int32_t elem;                    // bytes of an element
  bool l_wide;                     // L rows in 16-byte pieces
};

// Element offsets of token j of sequence t: its K / V row of head 0, and its L row's index.
__device__ __forceinline__ void gather_row(const GatherSide& c, int t, int j, int64_t& kv, int64_t& l) {
  if (c.block_size == 0) {
    kv = j * c.kv_token_stride;
    l = j;
    return;
  }
  const int blk = c.block_table[static_cast<int64_t>(t) * c.max_blocks_per_seq + (j >> 4)];
  kv = blk * c.kv_block_stride + (j & 15) * c.kv_token_stride;
  l = static_cast<int64_t>(blk) * 16 + (j & 15);
}

// One workgroup per sixteen new rows of a sequence and K or V (z), all heads: a memory-bound copy of 16-byte pieces, eight
// in flight per lane, piece fastest, then the row, then the head, so that the rows of a destination block are written
// end to end.  The workgroups of K move the L rows and the weights as well.
__global__ __launch_bounds__(256) void cache_gather_kernel(GatherParams p) {
  __shared__ int64_t kv_s[2][16], l_s[2][16];
  const int t = blockIdx.y, i0 = blockIdx.x * 16;
  const int rows = min(16, min(p.new_lens[t], p.dst.max_seq_len) - i0);
  if (rows <= 0) return;
  const int tid = threadIdx.x;
  if (tid < 32) {
    const int r = min(tid & 15, rows - 1), side = tid >> 4;
    const int from = min(max(p.kept[t * p.kept_stride + i0 + r], 0), p.src.max_seq_len - 1);
    int64_t kv, l;
    if (side == 0) gather_row(p.src, t, from, kv, l);
    else gather_row(p.dst, t, i0 + r, kv, l);
    kv_s[side][tid & 15] = kv * p.elem;
    l_s[side][tid & 15] = l;
    if (blockIdx.z == 0 && side == 0 && p.weights != nullptr && (tid & 15) < rows)
      p.dst_weights[t * p.dst_weights_stride + i0 + r] = p.weights[t * p.weights_stride + from];
  }
  __syncthreads();
  const char* src = static_cast<const char*>(blockIdx.z == 0 ? p.src.k : p.src.v);
  char* dst = static_cast<char*>(blockIdx.z == 0 ? p.dst.k : p.dst.v);
  const int64_t src_head = p.src.kv_head_stride * p.elem, dst_head = p.dst.kv_head_stride * p.elem;
  const int pcs = __builtin_ctz(p.row_pieces), total = p.n_kv_heads * 16 * p.row_pieces;  // (8, 16 or 32 pieces)
  constexpr int U = 8;
  for (int e0 = tid; e0 < total; e0 += 256 * U) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (past the end: a piece that is there, read again)
      const int e = min(e0 + 256 * u, total - 1), c = e & (p.row_pieces - 1), r = (e >> pcs) & 15, h = e >> (pcs + 4);
      v[u] = *reinterpret_cast<const u32x4*>(src + kv_s[0][r] + h * src_head + c * 16);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + 256 * u, c = e & (p.row_pieces - 1), r = (e >> pcs) & 15, h = e >> (pcs + 4);
      if (e < total && r < rows) *reinterpret_cast<u32x4*>(dst + kv_s[1][r] + h * dst_head + c * 16) = v[u];
    }
  }
  if (blockIdx.z != 0) return;
  for (int a = 0; a < p.n_adapters; ++a) {
    const char* from = static_cast<const char*>(p.src.l) + a * p.src.l_adapter_stride * p.elem;
    char* to = static_cast<char*>(p.dst.l) + a * p.dst.l_adapter_stride * p.elem;
    const int64_t fs = p.src.l_row_stride * p.elem, ts = p.dst.l_row_stride * p.elem;
    if (p.l_wide) {
      const int per = p.l_bytes >> 4;  // at most sixteen
      for (int e = tid; e < rows * per; e += 256) {
        const int r = e / per, c = e - r * per;
        *reinterpret_cast<uint4*>(to + l_s[1][r] * ts + c * 16) = *reinterpret_cast<const uint4*>(from + l_s[0][r] * fs + c * 16);
      }
    } else {
      const int per = p.l_bytes >> 1;  // (rows of any rank: two bytes at a time)
      for (int e = tid; e < rows * per; e += 256) {
        const int r = e / per, c = e - r * per;
        *reinterpret_cast<uint16_t*>(to + l_s[1][r] * ts + c * 2) = *reinterpret_cast<const uint16_t*>(from + l_s[0][r] * fs + c * 2);
      }
    }
  }
}

static GatherSide gather_side(const lra_shape* sh, const lra_cache* c) {
  GatherSide s{};
  s.k = const_cast<void*>(c->k_base);
  s.v = const_cast<void*>(c->v_base);
  s.l = const_cast<void*>(c->l);
  s.block_table = c->block_table;
  s.kv_token_stride = c->kv_token_stride;
  s.kv_head_stride = c->kv_head_stride;
  s.kv_block_stride = c->kv_block_stride;
  s.l_row_stride = c->l_row_stride ? c->l_row_stride : sh->rank;
  s.l_adapter_stride = c->l_adapter_stride;
  s.block_size = c->block_size;
  s.max_blocks_per_seq = c->max_blocks_per_seq;
  s.max_seq_len = c->max_seq_len;
  return s;
}

}  // namespace lra

using namespace lra;

extern "C" {

lra_status lra_evict_select(const lra_cache* cache, const float* weights, int64_t weights_stride, int32_t budget, int32_t sinks,
                            int32_t recent, int32_t* kept, int64_t kept_stride, int32_t* new_lens, void* stream) {
  if (!cache || !cache->seq_lens || !weights || !kept || !new_lens) return LRA_ERR_NULL;
  if (cache->n_seqs < 1 || cache->max_seq_len < 1) return LRA_ERR_SHAPE;
  if (cache->n_seqs > (1 << 20) || cache->max_seq_len > (1 << 30)) return LRA_ERR_UNSUPPORTED;
  if (budget < 1 || sinks < 0 || recent < 0 || static_cast<int64_t>(sinks) + recent > budget) return LRA_ERR_SHAPE;
  if (weights_stride < cache->max_seq_len || kept_stride < (budget < cache->max_seq_len ? budget : cache->max_seq_len)) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(new_lens)) & 3) return LRA_ERR_SHAPE;
  SelectParams p{};
  p.seq_lens = cache->seq_lens;
  p.weights = weights;
  p.kept = kept;
  p.new_lens = new_lens;
  p.weights_stride = weights_stride;
  p.kept_stride = kept_stride;
  p.max_seq_len = cache->max_seq_len;
  p.budget = budget;
  p.sinks = sinks;
  p.recent = recent;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(cache->n_seqs), block(1024);
  const int between = cache->max_seq_len - sinks - recent;  // (at most 2^30 less something, at least -2^31 + 1)
  if (between <= 4 * 1024) hipLaunchKernelGGL((evict_select_kernel<4>), grid, block, 0, s, p);
  else if (between <= 16 * 1024) hipLaunchKernelGGL((evict_select_kernel<16>), grid, block, 0, s, p);
  else if (between <= 64 * 1024) hipLaunchKernelGGL((evict_select_kernel<64>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((evict_select_kernel<0>), grid, block, 0, s, p);
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

lra_status lra_cache_gather(const lra_shape* shape, const lra_cache* src, int32_t n_adapters, const int32_t* kept, int64_t kept_stride,
                            const lra_cache* dst, const float* weights, int64_t weights_stride, float* dst_weights,
                            int64_t dst_weights_stride, void* stream) {
  lra_status st = check_common(shape, src);
  if (st != LRA_OK) return st;
  st = check_common(shape, dst);
  if (st != LRA_OK) return st;
  if (!kept || (weights == nullptr) != (dst_weights == nullptr)) return LRA_ERR_NULL;
  if (src->n_seqs != dst->n_seqs || n_adapters < 1 || kept_stride < dst->max_seq_len) return LRA_ERR_SHAPE;
  if (n_adapters > 1 && (src->l_adapter_stride == 0 || dst->l_adapter_stride == 0)) return LRA_ERR_SHAPE;
  if (weights && (weights_stride < src->max_seq_len || dst_weights_stride < dst->max_seq_len)) return LRA_ERR_SHAPE;
  if (weights && weights == dst_weights) return LRA_ERR_SHAPE;  // (workgroups would overwrite what others have yet to read)
  if (src->block_size == 0 ? src->k_base == dst->k_base || src->v_base == dst->v_base || src->l == dst->l
                           : dst->block_size != 0 && src->block_table == dst->block_table && src->k_base == dst->k_base)
    return LRA_ERR_SHAPE;
  if (shape->key_rope_theta > 0.f || src->n_seqs > 65535 || dst->max_seq_len > (1 << 27)) return LRA_ERR_UNSUPPORTED;
  GatherParams p{};
  p.src = gather_side(shape, src);
  p.dst = gather_side(shape, dst);
  p.kept = kept;
  p.new_lens = dst->seq_lens;
  p.weights = weights;
  p.dst_weights = dst_weights;
  p.kept_stride = kept_stride;
  p.weights_stride = weights_stride;
  p.dst_weights_stride = dst_weights_stride;
  p.n_kv_heads = shape->n_kv_heads;
  p.elem = shape->dtype == LRA_BF16 ? 2 : 4;
  p.row_pieces = shape->head_dim * p.elem / 16;
  p.l_bytes = shape->rank * p.elem;
  p.n_adapters = n_adapters;
  p.l_wide = (p.l_bytes | (p.src.l_row_stride * p.elem) | (p.dst.l_row_stride * p.elem)) % 16 == 0;
  hipLaunchKernelGGL(cache_gather_kernel, dim3((dst->max_seq_len + 15) / 16, dst->n_seqs, 2), dim3(256), 0,
                     static_cast<hipStream_t>(stream), p);
  return hipGetLastError() == hipSuccess ? LRA_OK : LRA_ERR_HIP;
}

}  // extern "C"
