// Fuzz driver for the checks and the planning of the 8-bit calls (csrc/lra_attn8_plan.cpp), built for the CPU alone with
// -fsanitize=address,undefined by tests/test_attn8_plan_sanitized.py: sizes up to and beyond the documented caps go through the
// argument checks and, where those accept them, through the planner, whose plans must keep their invariants.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "lra_attn8_plan.h"

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

#define CHECK(cond)                                                                                   \
  do {                                                                                                \
    if (!(cond)) {                                                                                    \
      std::fprintf(stderr, "attn8_plan_fuzz: %s failed at case %d (line %d)\n", #cond, it, __LINE__); \
      return 1;                                                                                       \
    }                                                                                                 \
  } while (0)

int main(int argc, char** argv) {
  const int cases = argc > 1 ? std::atoi(argv[1]) : 200000;
  alignas(16) static char dummy[64];
  const int32_t* ints = reinterpret_cast<const int32_t*>(dummy);
  int accepted = 0, few[5] = {}, tiles = 0, whole = 0, vector = 0, refused = 0, rows_taken = 0, by_length = 0, ordered = 0, shared = 0;
  for (int it = 0; it < cases; ++it) {
    lra_shape sh{};
    sh.n_kv_heads = static_cast<int32_t>(pick({1, 2, 4, 8, 3, 256}));
    sh.n_q_heads = sh.n_kv_heads * static_cast<int32_t>(pick({1, 2, 4, 7, 8, 16}));
    sh.head_dim = static_cast<int32_t>(pick({64, 128}));
    sh.rank = static_cast<int32_t>(pick({1, 8, 12, 16, 24, 32, 64}));
    sh.dtype = rnd() % 4 ? LRA_BF16 : LRA_F32;
    lra_cache8 c{};
    c.k = c.v = c.l = dummy;
    c.k_scale = c.v_scale = reinterpret_cast<uint8_t*>(dummy);
    c.seq_lens = ints;
    c.code = static_cast<int32_t>(rnd() % 2);
    c.max_seq_len = static_cast<int32_t>(upto(31));
    c.kv_head_stride = 16 * sh.head_dim + 16 * (upto(40) - 1);
    c.kv_block_stride = rnd() % 2 ? c.kv_head_stride * sh.n_kv_heads : 16 * upto(38);
    c.scale_block_stride = rnd() % 2 ? 0 : upto(33);
    c.l_row_stride = rnd() % 2 ? 0 : (sh.rank + 7) / 8 * 8 * upto(22);
    c.n_seqs = rnd() % 3 ? static_cast<int32_t>(upto(20)) : 1;
    if (rnd() % 4) c.block_table = ints;
    c.max_blocks_per_seq = static_cast<int32_t>(c.max_seq_len / 16 + upto(3) - 1);
    c.num_blocks = static_cast<int32_t>(rnd() % 2 ? c.max_blocks_per_seq : upto(30));
    lra_batch b{};
    b.seq_query_start = b.query_adapter = ints;
    b.n_queries = static_cast<int32_t>(upto(30));
    b.max_queries_per_seq = static_cast<int32_t>(rnd() % 2 ? upto(5) : upto(30));
    b.causal = rnd() % 2;
    b.window = rnd() % 2 ? 0 : static_cast<int32_t>(rnd() % 8 ? upto(30) : INT32_MAX);
    b.sinks = rnd() % 2 ? 0 : static_cast<int32_t>(rnd() % 8 ? upto(30) : INT32_MAX);
    lra_tuning user{};
    user.kernel_variant = static_cast<int32_t>(rnd() % 3);
    lra_new_rows n{};
    n.k = n.v = dummy;
    n.seq_start = ints;
    n.n_new = static_cast<int32_t>(upto(30));
    n.max_new_per_seq = static_cast<int32_t>(upto(30));
    n.k_token_stride = n.v_token_stride = static_cast<int64_t>(sh.n_kv_heads) * sh.head_dim + 16 * (upto(30) - 1);
    if (check_new_rows(&sh, &c, &n) == LRA_OK) ++rows_taken;
    if (check_batch8(&sh, &c, &b) != LRA_OK) {
      ++refused;
      continue;
    }
    ++accepted;
    const int64_t rows = static_cast<int64_t>(b.n_queries) * sh.n_q_heads, group = sh.n_q_heads / sh.n_kv_heads;
    const Attn8Plan pl = plan_attn8(&sh, &c, &b, resolve_tuning(&user));
    CHECK(pl.rows == rows);
    if (!pl.launchable) continue;
    CHECK(pl.n_splits >= 1 && pl.n_splits <= 64 && !(pl.few_rows && pl.tiles));
    const bool mfma = sh.dtype == LRA_BF16 && sh.rank % 8 == 0;
    if (pl.states) {
      const size_t states = static_cast<size_t>(rows) * static_cast<size_t>(pl.n_splits);
      CHECK(pl.off_ml + states * 8 <= pl.off_o && pl.off_o + states * static_cast<size_t>(sh.head_dim) * 4 <= pl.off_lr);
      CHECK(pl.off_lr + states * static_cast<size_t>(sh.rank) * 4 <= pl.off_adapter && pl.off_adapter + static_cast<size_t>(rows) * 4 <= pl.bytes);
    } else {
      CHECK(pl.bytes == 0 && pl.tiles && pl.n_splits == 1 && b.causal);
      ++whole;
    }
    if (pl.few_rows) {
      // every row of a sequence has a place in its workgroup
      ++few[pl.row_tiles];
      CHECK(mfma && (pl.row_tiles == 1 || pl.row_tiles == 2 || pl.row_tiles == 4));
      CHECK(c.n_seqs <= 65535 && b.max_queries_per_seq * group <= 16 * pl.row_tiles);
      CHECK(static_cast<int64_t>(sh.n_kv_heads) * pl.n_splits * 256 < (int64_t{1} << 32));
      if (pl.head_shares > 0) {  // (by the sequences' lengths)
        ++by_length;
        const int64_t most = pl.head_shares + c.n_seqs;
        CHECK(c.n_seqs > 1 && c.n_seqs <= kShareSeqs && pl.share_least >= 1 && pl.n_splits >= 1);
        CHECK(static_cast<int64_t>(sh.n_kv_heads) * ((most + 7) / 8 * 8) * 256 < (int64_t{1} << 32));
      }
    } else if (pl.tiles) {
      ++tiles;
      CHECK(pl.head_shares == 0 || (pl.n_splits > 1 && c.n_seqs > 1 && c.n_seqs <= kShareSeqs));
      CHECK(!pl.longest_first || (pl.n_splits == 1 && c.n_seqs > 1 && c.n_seqs <= kShareSeqs));
      ordered += pl.longest_first;
      shared += pl.head_shares > 0;
      CHECK(mfma && pl.tile_places >= (b.n_queries * group + 127) / 128 && pl.tile_places >= c.n_seqs);
      CHECK(static_cast<int64_t>(pl.tile_places) * sh.n_kv_heads * 256 < (int64_t{1} << 32));
    } else {
      ++vector;
      CHECK(pl.states && rows * 256 < (int64_t{1} << 32));
    }
  }
  if (!few[1] || !few[2] || !few[4] || !tiles || !whole || !vector || !refused || !rows_taken || !by_length || !ordered || !shared) {
    std::fprintf(stderr, "attn8_plan_fuzz: a kind of plan never came up (%d %d %d %d %d %d %d %d %d %d %d)\n", few[1], few[2], few[4], tiles, whole, vector,
                 refused, rows_taken, by_length, ordered, shared);
    return 1;
  }
  std::printf("%d accepted, all plans consistent\n", accepted);
  return 0;
}
