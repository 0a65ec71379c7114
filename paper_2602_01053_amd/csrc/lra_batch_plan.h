// Host-side checks and launch planning of the batch entry points.  Plain C++ with no HIP dependency, like lra_plan.h.
#pragma once

#include "lra_plan.h"

namespace lra {

lra_status check_batch(const lra_shape* sh, const lra_cache* c, const lra_batch* b);

struct BatchPlan {
  bool few_rows;   // batch_rows_kernel
  bool tiles;      // batch_tiles_kernel; neither: the vector-ALU kernels
  int tile_places; // ... and its q tiles per kv head,
  bool tile_per_query;  // ... of one query each
  bool states;     // the shares of a row leave states for the merge kernel
  int rows;        // n_queries x Hq
  int split_keys;  // vector-ALU kernels: keys per share, of those that a row sees
  int n_splits;
  size_t off_ml, off_o, off_lr, off_adapter, bytes;
  bool launchable;  // false: LRA_ERR_UNSUPPORTED
};
// key_adapter: whether the call has a B_K (without one a rotary key side has nothing to rotate).  lra_batch_workspace_bytes cannot
// know and tells the larger need of the two.
BatchPlan plan_batch(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune, bool key_adapter = true);
// 0 bytes is a valid need, (size_t)-1: neither call can be launched.
size_t batch_workspace_bytes(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune);

// lra_key_weights: the query rows' Q B_K^T and softmax statistics, then the sums over rows key by key.
struct WeightsPlan {
  bool mfma;     // else the vector-ALU kernels
  int n_splits;  // key shares of the statistics
  int tile_places;  // MFMA: places of 128 rows per kv head
  int rows;
  int sum_groups;   // MFMA, many rows: groups of kv heads that sum on their own
  size_t off_qt, off_lse, off_stats, off_sums, bytes;
};
WeightsPlan plan_key_weights(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune);

}  // namespace lra
