#include "lra_batch_plan.h"

#include <algorithm>

namespace lra {

lra_status check_batch(const lra_shape* sh, const lra_cache* c, const lra_batch* b) {
  const lra_status st = check_common(sh, c);
  if (st != LRA_OK) return st;
  if (!b || !b->seq_query_start || !b->query_adapter) return LRA_ERR_NULL;
  if (b->n_queries < 1 || b->max_queries_per_seq < 1 || b->max_queries_per_seq > b->n_queries) return LRA_ERR_SHAPE;
  if (b->window < 0 || b->sinks < 0) return LRA_ERR_SHAPE;
  if (static_cast<int64_t>(b->n_queries) * sh->n_q_heads > (int64_t{1} << 30)) return LRA_ERR_UNSUPPORTED;
  return LRA_OK;
}

static size_t aligned(size_t bytes) { return (bytes + 255) & ~static_cast<size_t>(255); }

// The most keys that one query sees.
static int64_t keys_per_row(const lra_cache* c, const lra_batch* b) {
  return b->window > 0 ? std::min<int64_t>(c->max_seq_len, static_cast<int64_t>(b->window) + b->sinks) : c->max_seq_len;
}

BatchPlan plan_batch(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune) {
  BatchPlan pl{};
  const int64_t rows = static_cast<int64_t>(b->n_queries) * sh->n_q_heads;
  const int64_t keys = keys_per_row(c, b);
  // vector-ALU kernels: one workgroup per row and share, three to a compute unit; a share of 256 keys at least, so
  // that its loop is longer than what stands around it
  int64_t share = tune.split_keys;
  if (share <= 0) {
    const int64_t shares = std::max<int64_t>(1, 3 * kCUs / rows);
    share = std::max<int64_t>((keys + shares - 1) / shares, 256);
  }
  share = std::min<int64_t>((share + 63) / 64 * 64, int64_t{1} << 30);
  pl.rows = static_cast<int>(rows);
  pl.split_keys = static_cast<int>(share);
  const int64_t splits = (keys + share - 1) / share;
  const bool rotary = sh->key_rope_theta > 0.f;
  pl.launchable = splits <= 65535 && (!rotary || rows < (int64_t{1} << 26));  // (a grid dimension holds fewer than 2^32 threads)
  if (!pl.launchable) return pl;
  pl.n_splits = static_cast<int>(splits);
  const size_t states = static_cast<size_t>(rows) * static_cast<size_t>(splits);
  pl.off_ml = 0;
  pl.off_o = aligned(states * 2 * sizeof(float));
  pl.off_lr = pl.off_o + aligned(states * sh->head_dim * sizeof(float));
  pl.off_adapter = pl.off_lr + aligned(states * sh->rank * sizeof(float));
  pl.bytes = pl.off_adapter + aligned(static_cast<size_t>(rows) * sizeof(int32_t));
  return pl;
}

WeightsPlan plan_key_weights(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune) {
  (void)c;
  (void)tune;
  WeightsPlan pl{};
  pl.rows = b->n_queries * sh->n_q_heads;  // (checked: at most 2^30)
  pl.off_qt = 0;
  pl.off_lse = aligned(static_cast<size_t>(pl.rows) * sh->rank * sizeof(float));
  pl.bytes = pl.off_lse + aligned(static_cast<size_t>(pl.rows) * sizeof(float));
  return pl;
}

}  // namespace lra
