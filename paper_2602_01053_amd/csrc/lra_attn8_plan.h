// Host-side argument checks and launch planning of the 8-bit calls (lra_attn8.h); plain C++ like lra_plan.h.
#pragma once

#include "lra_attn8.h"
#include "lra_plan.h"

namespace lra {

lra_status check_cache8(const lra_shape* sh, const lra_cache8* c);
lra_status check_batch8(const lra_shape* sh, const lra_cache8* c, const lra_batch* b);
lra_status check_new_rows(const lra_shape* sh, const lra_cache8* c, const lra_new_rows* n);

// The most sequences whose key shares the kernels for few rows form by their lengths.
constexpr int kShareSeqs = 128;

struct Attn8Plan {
  bool launchable;
  bool few_rows, tiles, states, longest_first;
  int rows, n_splits, row_tiles, tile_places;
  int head_shares, share_least;  // shares of a kv head over all sequences, by their lengths (0: n_splits of each); few rows: tiles of the shortest
  size_t off_ml, off_o, off_lr, off_adapter, bytes;
};
Attn8Plan plan_attn8(const lra_shape* sh, const lra_cache8* c, const lra_batch* b, const Tuning& tune);

}  // namespace lra
