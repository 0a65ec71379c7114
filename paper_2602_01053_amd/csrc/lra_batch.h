// Batches of queries with a window (lra_batch of the header): kernel parameters and what a query sees.
#pragma once

#include "lra_attn.h"
#include "lra_common.h"

namespace lra {

// (fields of its own block: longer parameters would move those of the other kernels)
struct BatchParams : Params {
  int32_t causal, window, sinks;
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

// Whether a query at position pos sees token j.
__device__ __forceinline__ bool batch_sees(const BatchParams& p, int pos, int j) {
  return j <= pos && (p.window == 0 || j > pos - p.window || j < p.sinks);
}

// Parameters of a call out of the ABI's structs (pointers of the workspace and of the outputs left NULL).
BatchParams batch_params(const lra_shape* sh, const lra_cache* c, const lra_adapters* ad, const lra_batch* b, const void* q);

hipError_t launch_batch_partials(const BatchParams& p, bool is_bf16, int rows, hipStream_t s);
// States of n_splits key shares per row -> out; rows without any give zeros
hipError_t launch_batch_merge(const BatchParams& p, bool is_bf16, int rows, hipStream_t s);

}  // namespace lra
