// What the planner of the batch calls answers for one call (tests/test_batch_plan_cpu.py).
#include "lra_batch_plan.h"

extern "C" void batch_plan_query(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const lra_tuning* tuning, int key_adapter,
                                 int32_t* out) {
  const lra::BatchPlan pl = lra::plan_batch(sh, c, b, lra::resolve_tuning(tuning), key_adapter != 0);
  out[0] = pl.few_rows;
  out[1] = pl.tiles;
  out[2] = pl.tile_places;
  out[3] = pl.tile_per_query;
  out[4] = pl.states;
  out[5] = pl.n_splits;
  out[6] = pl.split_keys;
  out[7] = pl.launchable;
  out[8] = static_cast<int32_t>(pl.bytes >> 8);
}

extern "C" int32_t batch_workspace_query(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const lra_tuning* tuning) {
  return static_cast<int32_t>(lra::batch_workspace_bytes(sh, c, b, lra::resolve_tuning(tuning)) >> 8);
}

extern "C" void weights_plan_query(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const lra_tuning* tuning, int32_t* out) {
  const lra::WeightsPlan pl = lra::plan_key_weights(sh, c, b, lra::resolve_tuning(tuning));
  out[0] = pl.mfma;
  out[1] = pl.n_splits;
  out[2] = pl.tile_places;
  out[3] = pl.sum_groups;
}
