// Fuzz driver for the planning of lra_attn_batch and lra_key_weights (csrc/lra_batch_plan.cpp), built for the CPU alone with
// -fsanitize=address,undefined by tests/test_batch_plan_sanitized.py: sizes up to and beyond the documented caps go through
// the argument checks and, where those accept them, through the planner, whose plans must keep their invariants.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "lra_batch_plan.h"

using namespace lra;

static uint64_t state = 0x9e3779b97f4a7c15ull;
static uint64_t rnd() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return state;
}
static int64_t pick(std::initializer_list<int64_t> v) { return *(v.begin() + rnd() % v.size()); }
static int64_t upto(int log2) { return static_cast<int64_t>(rnd() % (uint64_t{1} << (1 + rnd() % log2))) + 1; }

#define CHECK(cond)                                                                                       \
  do {                                                                                                    \
    if (!(cond)) {                                                                                        \
      std::fprintf(stderr, "batch_plan_fuzz: %s failed at case %d (line %d)\n", #cond, it, __LINE__);     \
      return 1;                                                                                           \
    }                                                                                                     \
  } while (0)

int main(int argc, char** argv) {
  const int cases = argc > 1 ? std::atoi(argv[1]) : 200000;
  static char dummy[64];
  const int32_t* ints = reinterpret_cast<const int32_t*>(dummy);
  int accepted = 0, few = 0, tiles = 0, vector = 0, mfma_weights = 0, divided = 0;
  for (int it = 0; it < cases; ++it) {
    lra_shape sh{};
    sh.n_kv_heads = static_cast<int32_t>(pick({1, 2, 4, 8, 3, 256}));
    sh.n_q_heads = sh.n_kv_heads * static_cast<int32_t>(pick({1, 2, 4, 7, 8, 16}));
    sh.head_dim = static_cast<int32_t>(pick({64, 128}));
    sh.rank = static_cast<int32_t>(pick({1, 8, 12, 16, 24, 32, 64}));
    sh.dtype = rnd() % 4 ? LRA_BF16 : LRA_F32;
    sh.key_rope_theta = rnd() % 4 ? 0.f : 500000.f;
    lra_cache c{};
    c.k_base = c.v_base = c.l = dummy;
    c.seq_lens = ints;
    c.max_seq_len = static_cast<int32_t>(upto(30));
    c.kv_token_stride = sh.head_dim + 8 * (upto(3) - 1);
    c.kv_head_stride = c.kv_token_stride * 16;
    c.n_seqs = 1;
    if (rnd() % 3) {
      c.block_size = 16;
      c.block_table = ints;
      c.n_seqs = static_cast<int32_t>(upto(20));
      c.max_blocks_per_seq = (c.max_seq_len + 15) / 16 + static_cast<int32_t>(upto(3));
      c.num_blocks = static_cast<int32_t>(upto(30));
      c.kv_block_stride = c.kv_head_stride * sh.n_kv_heads;
    }
    c.l_row_stride = rnd() % 2 ? 0 : (sh.rank + 7) / 8 * 8 * upto(3);
    c.l_adapter_stride = rnd() % 4 ? 0 : 8 * upto(36);
    lra_batch b{};
    b.seq_query_start = b.query_adapter = ints;
    b.n_queries = static_cast<int32_t>(upto(30));
    b.max_queries_per_seq = static_cast<int32_t>(rnd() % 2 ? upto(5) : upto(30));
    b.causal = rnd() % 2;
    b.window = rnd() % 2 ? 0 : static_cast<int32_t>(rnd() % 8 ? upto(30) : INT32_MAX);
    b.sinks = rnd() % 2 ? 0 : static_cast<int32_t>(rnd() % 8 ? upto(30) : INT32_MAX);
    lra_tuning user{};
    user.kernel_variant = static_cast<int32_t>(rnd() % 3);
    user.decode_split_keys = rnd() % 4 ? 0 : static_cast<int32_t>(upto(30));
    if (check_batch(&sh, &c, &b) != LRA_OK) continue;
    ++accepted;
    const Tuning tune = resolve_tuning(&user);
    const int64_t rows = static_cast<int64_t>(b.n_queries) * sh.n_q_heads;

    const BatchPlan pl = plan_batch(&sh, &c, &b, tune);
    CHECK(pl.rows == rows);
    if (pl.launchable) {
      CHECK(pl.n_splits >= 1 && pl.n_splits <= 65535);
      CHECK(!(pl.few_rows && pl.tiles));
      if (pl.states) {
        const size_t states = static_cast<size_t>(rows) * static_cast<size_t>(pl.n_splits);
        CHECK(pl.off_ml + states * 8 <= pl.off_o && pl.off_o + states * static_cast<size_t>(sh.head_dim) * 4 <= pl.off_lr);
        CHECK(pl.off_lr + states * static_cast<size_t>(sh.rank) * 4 <= pl.off_adapter && pl.off_adapter + static_cast<size_t>(rows) * 4 <= pl.bytes);
      } else {
        CHECK(pl.bytes == 0 && pl.tiles && pl.n_splits == 1);
      }
      if (pl.few_rows) {
        ++few;
        CHECK(c.n_seqs <= 65535 && b.max_queries_per_seq * (sh.n_q_heads / sh.n_kv_heads) <= 32 && pl.n_splits <= 64);
      } else if (pl.tiles) {
        ++tiles;
        CHECK(pl.n_splits <= 64 && pl.tile_places >= 1 && static_cast<int64_t>(pl.tile_places) * sh.n_kv_heads * 256 < (int64_t{1} << 32));
        const int64_t group = sh.n_q_heads / sh.n_kv_heads;
        CHECK(pl.tile_places >= (pl.tile_per_query ? b.n_queries : (b.n_queries * group + 127) / 128));
      } else {
        ++vector;
        CHECK(pl.split_keys >= 1);
      }
    }
    if (c.n_seqs > 65535) continue;
    const WeightsPlan w = plan_key_weights(&sh, &c, &b, tune);
    CHECK(w.rows == rows && w.n_splits >= 1 && w.n_splits <= 32);
    CHECK(w.off_qt <= w.off_lse && w.off_lse <= w.off_stats && w.off_stats + static_cast<size_t>(rows) * static_cast<size_t>(w.n_splits) * 8 <= w.bytes);
    if (w.mfma) {
      ++mfma_weights;
      CHECK(w.sum_groups >= 1 && w.sum_groups <= sh.n_kv_heads);
      CHECK(static_cast<int64_t>(w.tile_places) * w.n_splits * sh.n_kv_heads * 256 < (int64_t{1} << 32));
      if (w.sum_groups > 1) {
        ++divided;
        const size_t sums = static_cast<size_t>(w.sum_groups) * static_cast<size_t>(c.n_seqs) * static_cast<size_t>(c.max_seq_len) * 4;
        CHECK(w.off_sums + sums <= w.bytes && sums <= size_t{1} << 22);
      }
    }
  }
  if (!few || !tiles || !vector || !mfma_weights || !divided) {
    std::fprintf(stderr, "batch_plan_fuzz: a kind of plan never came up (%d %d %d %d %d)\n", few, tiles, vector, mfma_weights, divided);
    return 1;
  }
  std::printf("%d accepted, all plans consistent\n", accepted);
  return 0;
}
