// Batches of queries with a window (lra_batch of the header): kernel parameters and what a query sees.
#pragma once

#include "lra_attn.h"
#include "lra_common.h"

namespace lra {

// (fields of its own block: longer parameters would move those of the other kernels)
struct BatchParams : Params {
  int32_t causal, window, sinks;
  int32_t tile_places;     // batch_tiles_kernel: places of q tiles per kv head (batch_places, or the queries)
  int32_t tile_per_query;  // ... whose tiles hold one query each
};

// Sequence of query `tok`: the last t with seq_query_start[t] <= tok.
__device__ __forceinline__ int sequence_of_query(const Params& p, int tok) {
  int lo = 0, hi = p.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.seq_query_start[mid] <= tok) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// What the query token `tok` sees of its sequence: n_keys tokens, numbered 0 .. n_keys - 1, of which the first
// n_sinks are the sequence's first and number k >= n_sinks is token k + gap.
struct BatchRow {
  int t, adapter, n_keys, n_sinks, gap;
};
__device__ __forceinline__ BatchRow batch_row(const BatchParams& p, int tok) {
  BatchRow b;
  b.t = p.n_seqs > 1 ? sequence_of_query(p, tok) : 0;
  const int first = b.t > 0 ? p.seq_query_start[b.t] : 0;
  const int end = b.t + 1 < p.n_seqs ? p.seq_query_start[b.t + 1] : p.n_queries;
  const int n_t = min(p.seq_lens[b.t], p.max_seq_len);
  const int pos = p.causal ? n_t - (end - tok) : n_t - 1;
  b.adapter = min(max(p.query_adapter[p.causal ? first : tok], 0), p.n_adapters - 1);
  const int lo = p.window > 0 ? max(0, pos - p.window + 1) : 0;
  b.n_sinks = min(p.sinks, lo);  // (zero without a window)
  b.gap = lo - b.n_sinks;
  b.n_keys = pos < 0 ? 0 : pos + 1 - b.gap;
  return b;
}

// The q tiles of a batch (lra_batch_tiles.h): 128 rows of one sequence's queries at most, a row being a query's token at one of
// the q heads of a kv head; or one query, where its adapter decides what the keys or their low-rank rows are.
struct BatchTiles {
  int t, n_t;
  int adapter;                 // of the first query: of all, where the call is causal or a tile holds one
  int first_query, n_queries;  // the queries of the chunk
  int first_pos;               // position of the first of them
  int tile;                    // of the chunk's tiles; past the last: nothing to do
};

// Sequence t takes ceil(c_t G / 128) tiles, and has the places from floor(start_t G / 128) + t on: at least as many, since
// floor(a + b) >= floor(a) + floor(b), and found without a running sum over the sequences.  Place `at` is looked for by the
// 64 lanes of a wave, sixty-four times fewer sequences a step.
__device__ __forceinline__ int batch_places(int n_queries, int group, int n_seqs) {
  return static_cast<int>((static_cast<int64_t>(n_queries) * group) >> 7) + n_seqs;
}
__device__ __forceinline__ BatchTiles batch_tiles(const BatchParams& p, int at, int lane) {
  BatchTiles b;
  if (p.tile_per_query) {
    b.t = p.n_seqs > 1 ? __builtin_amdgcn_readfirstlane(sequence_of_query(p, at)) : 0;
    b.first_query = at;
    b.n_queries = 1;
    b.tile = 0;
    b.n_t = __builtin_amdgcn_readfirstlane(min(p.seq_lens[b.t], p.max_seq_len));
    // (of a causal chunk it is one too, with its place in it)
    const int first = b.t > 0 ? p.seq_query_start[b.t] : 0, end = b.t + 1 < p.n_seqs ? p.seq_query_start[b.t + 1] : p.n_queries;
    b.first_pos = p.causal ? b.n_t - __builtin_amdgcn_readfirstlane(end - at) : b.n_t - 1;
    b.adapter = __builtin_amdgcn_readfirstlane(min(max(p.query_adapter[p.causal ? first : at], 0), p.n_adapters - 1));
    return b;
  }
  auto first_of = [&](int t) __attribute__((always_inline)) -> int {
    return t >= p.n_seqs ? p.n_queries : (t == 0 ? 0 : min(max(p.seq_query_start[t], 0), p.n_queries));
  };
  int lo = 0, cnt = p.n_seqs;
  while (cnt > 1) {
    const int step = (cnt + 63) >> 6;
    const int t = lo + lane * step;
    const bool before = t < lo + cnt && (t == lo || batch_places(first_of(t), p.group, t) <= at);
    const int k = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(before));
    cnt = min(step, lo + cnt - (lo + k * step));
    lo += k * step;
  }
  b.t = lo;
  b.first_query = __builtin_amdgcn_readfirstlane(first_of(lo));
  const int end = __builtin_amdgcn_readfirstlane(first_of(lo + 1));
  b.n_queries = max(0, end - b.first_query);
  b.tile = at - batch_places(b.first_query, p.group, lo);
  b.n_t = __builtin_amdgcn_readfirstlane(min(p.seq_lens[lo], p.max_seq_len));
  b.first_pos = p.causal ? b.n_t - b.n_queries : b.n_t - 1;
  b.adapter = b.n_queries > 0 ? __builtin_amdgcn_readfirstlane(min(max(p.query_adapter[b.first_query], 0), p.n_adapters - 1)) : 0;
  return b;
}
// Whether a query at position pos sees token j.
__device__ __forceinline__ bool batch_sees(const BatchParams& p, int pos, int j) {
  return j <= pos && (p.window == 0 || j > pos - p.window || j < p.sinks);
}

// A tile's (or a lane's) largest score in base-2 units; one below -2^30 (a mask of the type's lowest value) counts as minus infinity: as a reference, its
// rounding alone would be more than exp2 of the differences to it can hold.
__device__ __forceinline__ float tile_reference(float mx) { return mx < -0x1p30f ? -INFINITY : mx; }

// Parameters of a call out of the ABI's structs (pointers of the workspace and of the outputs left NULL).
BatchParams batch_params(const lra_shape* sh, const lra_cache* c, const lra_adapters* ad, const lra_batch* b, const void* q);

// part_ml NULL: no states, the outputs themselves (n_splits 1)
hipError_t launch_batch_tiles_d64(const BatchParams& p, hipStream_t s);
hipError_t launch_batch_tiles_d128(const BatchParams& p, hipStream_t s);
hipError_t launch_batch_rows(const BatchParams& p, hipStream_t s);
// The partial kernels' states go to the merge kernels of every other call (launch_merge), which divide by the row sum: a row that
// sees nothing has the state m = 0, l = 1, O = 0, O_lr = 0 in its first share.
hipError_t launch_batch_partials(const BatchParams& p, bool is_bf16, int rows, hipStream_t s);

}  // namespace lra
