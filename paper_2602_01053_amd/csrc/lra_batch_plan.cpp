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

// Whether the MFMA kernels can address the caches: a contiguous kv head's rows (or a block's), and the low-rank rows of one adapter, by
// 32-bit byte offsets inside one buffer resource, below the offset that stands for "outside" (2^31).
static bool mfma_fits(const lra_shape* sh, const lra_cache* c) {
  const int64_t lim = (int64_t{1} << 31) - 4096;
  const int64_t pitch = c->l_row_stride ? c->l_row_stride : sh->rank;
  const int64_t l_rows = c->block_size == 0 ? c->max_seq_len : static_cast<int64_t>(c->num_blocks) * 16;
  if (pitch > lim / 2 / l_rows) return false;
  return (c->block_size != 0 ? 16 : static_cast<int64_t>(c->max_seq_len)) * c->kv_token_stride * 2 <= lim;
}

static bool pool_fits(const lra_shape* sh, const lra_cache* c) {  // (prefill_pool_fits on the ABI's structs)
  const int64_t blocks = std::max(c->num_blocks, c->max_blocks_per_seq), lim = 0x7ffff000 / 2;
  return c->kv_block_stride <= lim / blocks && blocks * c->kv_block_stride + sh->n_kv_heads * c->kv_head_stride + 16 * c->kv_token_stride <= lim;
}

static void place_states(BatchPlan& pl, const lra_shape* sh) {
  // (the merge kernels: 128 to 1024 threads per row where there are more than 65535 queries)
  if (pl.rows / sh->n_q_heads > 65535 && static_cast<int64_t>(pl.rows) * (pl.n_splits <= 8 ? 128 : 1024) >= (int64_t{1} << 32)) {
    pl.launchable = false;
    return;
  }
  const size_t states = static_cast<size_t>(pl.rows) * static_cast<size_t>(pl.n_splits);
  pl.states = true;
  pl.off_ml = 0;
  pl.off_o = aligned(states * 2 * sizeof(float));
  pl.off_lr = pl.off_o + aligned(states * sh->head_dim * sizeof(float));
  pl.off_adapter = pl.off_lr + aligned(states * sh->rank * sizeof(float));
  pl.bytes = pl.off_adapter + aligned(static_cast<size_t>(pl.rows) * sizeof(int32_t));
}

// Key shares where a compute unit holds one workgroup (batch_tiles_kernel with a rotated key side at d = 128 and ranks above 32: some 420
// registers).  Units of about equal length: those with the shortest sum of turns, up to four of the chip, a turn being its key tiles and
// what a prologue takes, five tiles' time.  Sequences of any lengths: four turns' worth, so that the short ones' places go on to others,
// though beyond one turn's no share of less than ten tiles.
// (Planned as two workgroups to a unit, one turn: 333 new tokens of 28 heads behind a window of 1000, rank 64, 90 us against 77; 4 agents on
// 16 k tokens 119 against 107; 8 sequences of 1 k to 9 k, 4 agents, 446 against 366.  By turns whatever the lengths: the last 506.)
static int64_t shares_by_turns(int64_t units, int64_t key_tiles, bool ragged) {
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>((key_tiles + 1) / 2, 64));
  if (ragged) return std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(std::min<int64_t>(4 * kCUs / units, key_tiles / 10), kCUs / units), most));
  int64_t best = 1, least = INT64_MAX;
  for (int64_t s = 1; s <= most && (s == 1 || units * s <= 4 * kCUs); ++s) {
    const int64_t time = (units * s + kCUs - 1) / kCUs * ((key_tiles + s - 1) / s + 5);
    if (time < least) {
      least = time;
      best = s;
    }
  }
  return best;
}

// A workgroup of batch_tiles_kernel takes 128 rows of one sequence; where a query's adapter decides what the keys or their
// low-rank rows are (a rotated key side, a low-rank cache per adapter), and the queries of a sequence may have different ones,
// one query.  The key tiles of a q tile are shared where there are fewer q tiles than the chip has places, two per compute
// unit (but see shares_by_turns), and then so that they fill the places once; a share walks two tiles at least.
static bool plan_tiles(BatchPlan& pl, const lra_shape* sh, const lra_cache* c, const lra_batch* b, bool rotary) {
  const int64_t G = sh->n_q_heads / sh->n_kv_heads;
  pl.tile_per_query = !b->causal && (rotary || c->l_adapter_stride > 0);
  const int64_t places = pl.tile_per_query ? b->n_queries : b->n_queries * G / 128 + c->n_seqs;
  if (places * sh->n_kv_heads >= (int64_t{1} << 24)) return false;  // (a grid dimension holds fewer than 2^32 threads)
  const int64_t q_tiles = pl.tile_per_query ? b->n_queries : std::max<int64_t>((b->n_queries * G + 127) / 128, std::min(c->n_seqs, b->n_queries));
  const int64_t chunk = b->causal ? std::min<int64_t>(b->max_queries_per_seq, 128 / G + 1) : 1;
  const int64_t key_tiles = (std::min<int64_t>(c->max_seq_len, keys_per_row(c, b) + chunk) + 63) / 64 + (b->window > 0 ? 2 : 0);
  const int64_t units = q_tiles * sh->n_kv_heads;
  const bool one_per_unit = rotary && sh->head_dim == 128 && sh->rank > 32;
  // (a window of half the longest sequence or less: most see all of it)
  const bool ragged = c->n_seqs > 1 && 2 * keys_per_row(c, b) > c->max_seq_len;
  const int64_t shares = one_per_unit ? shares_by_turns(units, key_tiles, ragged)
                                      : std::max<int64_t>(1, std::min<int64_t>({2 * kCUs / units, (key_tiles + 1) / 2, 64}));
  pl.tiles = true;
  pl.tile_places = static_cast<int>(places);
  pl.n_splits = static_cast<int>(shares);
  // states also where the rows of a tile have adapters of their own (the merge kernel applies B_V row by row), and in the forms
  // that are built with them only
  const bool far = c->block_size != 0 && !pool_fits(sh, c);
  if (shares > 1 || far || rotary || (!b->causal && !pl.tile_per_query)) place_states(pl, sh);
  return true;
}

// 32 rows at most per sequence and kv head, with one low-rank cache: workgroups of (kv head, key share, sequence), two to a compute
// unit, whose waves have a tile of 32 keys each at least.
static bool plan_few_rows(BatchPlan& pl, const lra_shape* sh, const lra_cache* c, const lra_batch* b, bool rotary) {
  const int64_t G = sh->n_q_heads / sh->n_kv_heads;
  if (b->max_queries_per_seq * G > 32 || rotary || c->n_seqs > 65535) return false;
  if (c->l_adapter_stride > 0 && !b->causal) return false;  // (the rows of a sequence share their low-rank rows)
  const int64_t units = static_cast<int64_t>(sh->n_kv_heads) * std::min(c->n_seqs, b->n_queries);
  const int64_t chunk = b->causal ? b->max_queries_per_seq : 1;
  const int64_t key_tiles = (std::min<int64_t>(c->max_seq_len, keys_per_row(c, b) + chunk) + 31) / 32 + (b->window > 0 ? 2 : 0);
  pl.few_rows = true;
  pl.n_splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({2 * kCUs / units, (key_tiles + 3) / 4, 64})));
  place_states(pl, sh);
  return true;
}

BatchPlan plan_batch(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune, bool key_adapter) {
  BatchPlan pl{};
  const bool rotary = sh->key_rope_theta > 0.f && key_adapter;
  const int64_t rows = static_cast<int64_t>(b->n_queries) * sh->n_q_heads;
  const int64_t keys = keys_per_row(c, b);
  pl.rows = static_cast<int>(rows);
  pl.launchable = true;
  if (sh->dtype == LRA_BF16 && sh->rank % 8 == 0 && tune.variant != 1 && mfma_fits(sh, c)) {
    if (tune.variant == 0 && plan_few_rows(pl, sh, c, b, rotary)) return pl;
    if (plan_tiles(pl, sh, c, b, rotary)) return pl;
  }
  // vector-ALU kernels: one workgroup per row and share, three to a compute unit; a share of 256 keys at least, so
  // that its loop is longer than what stands around it
  int64_t share = tune.split_keys;
  if (share <= 0) {
    const int64_t shares = std::max<int64_t>(1, 3 * kCUs / rows);
    share = std::max<int64_t>((keys + shares - 1) / shares, 256);
  }
  share = std::min<int64_t>((share + 63) / 64 * 64, int64_t{1} << 30);
  pl.split_keys = static_cast<int>(share);
  const int64_t splits = (keys + share - 1) / share;
  pl.launchable = splits <= 65535 && (!rotary || rows < (int64_t{1} << 26));  // (a grid dimension holds fewer than 2^32 threads)
  if (!pl.launchable) return pl;
  pl.n_splits = static_cast<int>(splits);
  place_states(pl, sh);
  return pl;
}

size_t batch_workspace_bytes(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune) {
  const BatchPlan with = plan_batch(sh, c, b, tune, true), without = plan_batch(sh, c, b, tune, false);
  if (!with.launchable && !without.launchable) return static_cast<size_t>(-1);
  return std::max(with.launchable ? with.bytes : 0, without.launchable ? without.bytes : 0);
}

WeightsPlan plan_key_weights(const lra_shape* sh, const lra_cache* c, const lra_batch* b, const Tuning& tune) {
  WeightsPlan pl{};
  pl.rows = b->n_queries * sh->n_q_heads;  // (checked: at most 2^30)
  const size_t rows = static_cast<size_t>(pl.rows);
  pl.off_qt = 0;
  const int64_t G = sh->n_q_heads / sh->n_kv_heads;
  const int64_t places = b->n_queries * G / 128 + c->n_seqs;
  // statistics: workgroups of (kv head, 128 rows, share), three to a compute unit (two by registers at d = 128 and ranks above 32: planned as
  // three, 16 sequences of 4 agents took 455 us against 441, 100 rows of 18 k tokens 157 against 148), each with two 64-key tiles at least;
  // at most 32 shares, which the pass over them reads
  const int64_t q_tiles = std::max<int64_t>((b->n_queries * G + 127) / 128, std::min(c->n_seqs, b->n_queries));
  const int64_t tiles = (std::min<int64_t>(c->max_seq_len, keys_per_row(c, b) + (b->causal ? std::min<int64_t>(b->max_queries_per_seq, 128 / G + 1) : 1)) + 63) / 64 + 1;
  const int64_t per_unit = sh->head_dim == 128 && sh->rank > 32 ? 2 : 3;
  const int64_t shares = std::max<int64_t>(1, std::min<int64_t>({per_unit * kCUs / (q_tiles * sh->n_kv_heads), (tiles + 1) / 2, 32}));
  if (sh->dtype == LRA_BF16 && sh->rank % 8 == 0 && c->l_adapter_stride == 0 && tune.variant != 1 && mfma_fits(sh, c) &&
      places * shares * sh->n_kv_heads < (int64_t{1} << 24) && (b->n_queries * G + 63) / 64 < (int64_t{1} << 24)) {  // (weights_lse_kernel's)
    pl.mfma = true;
    pl.n_splits = static_cast<int>(shares);
    pl.tile_places = static_cast<int>(places);
    const size_t rp = sh->rank <= 16 ? 16 : (sh->rank <= 32 ? 32 : 64);
    pl.off_lse = aligned(rows * 2 * rp * 2);
    pl.off_stats = pl.off_lse + aligned(rows * sizeof(float));
    pl.off_sums = pl.bytes = pl.off_stats + aligned(rows * static_cast<size_t>(pl.n_splits) * 2 * sizeof(float));
    // sums over many rows: workgroups of 128 keys, the heads divided as long as all workgroups are on the chip at once, two to a
    // compute unit (64 queries, 18 k tokens, 8 heads: 29 us in 3 groups; 31 in 8, which come in three turns)
    const int64_t spans = static_cast<int64_t>(c->max_seq_len + 127) / 128 * c->n_seqs;
    pl.sum_groups = 1;
    if (b->max_queries_per_seq * G > 32) {
      pl.sum_groups = static_cast<int>(std::min<int64_t>(sh->n_kv_heads, std::max<int64_t>(1, 2 * kCUs / spans)));
      if (pl.sum_groups > 1)
        pl.bytes += aligned(static_cast<size_t>(pl.sum_groups) * static_cast<size_t>(c->n_seqs) * static_cast<size_t>(c->max_seq_len) * sizeof(float));
    }
    return pl;
  }
  // vector-ALU kernels: three workgroups to a compute unit, a share of 128 keys at least
  pl.n_splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({3 * kCUs / static_cast<int64_t>(rows), (keys_per_row(c, b) + 127) / 128, 32})));
  pl.off_lse = pl.off_stats = aligned(rows * sh->rank * sizeof(float));
  pl.bytes = pl.off_stats + aligned(rows * static_cast<size_t>(pl.n_splits) * 2 * sizeof(float));
  return pl;
}

}  // namespace lra
