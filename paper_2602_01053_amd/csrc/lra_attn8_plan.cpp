#include "lra_attn8_plan.h"

#include <algorithm>
#include <cmath>

namespace lra {

// What holds of a shape for every call, checked as for a paged cache of 16-bit rows.
static lra_status check_shape8(const lra_shape* sh) {
  if (sh->dtype != LRA_BF16 && sh->dtype != LRA_F32) return LRA_ERR_DTYPE;
  if (sh->n_q_heads < 1 || sh->n_kv_heads < 1 || sh->head_dim < 1 || sh->rank < 1) return LRA_ERR_SHAPE;
  if (sh->n_q_heads % sh->n_kv_heads) return LRA_ERR_SHAPE;
  if (!(sh->scale >= 0.f) || std::isinf(sh->scale)) return LRA_ERR_SHAPE;
  if (!(sh->key_rope_theta >= 0.f) || std::isinf(sh->key_rope_theta)) return LRA_ERR_SHAPE;
  if (sh->head_dim != 64 && sh->head_dim != 128) return LRA_ERR_UNSUPPORTED;
  if (sh->rank > 64 || sh->n_q_heads / sh->n_kv_heads > 16 || sh->n_q_heads > 4096) return LRA_ERR_UNSUPPORTED;
  return LRA_OK;
}

lra_status check_cache8(const lra_shape* sh, const lra_cache8* c) {
  if (!sh || !c) return LRA_ERR_NULL;
  const lra_status st = check_shape8(sh);
  if (st != LRA_OK) return st;
  if (c->code != LRA_E4M3 && c->code != LRA_INT8) return LRA_ERR_DTYPE;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->l || !c->seq_lens) return LRA_ERR_NULL;
  if (c->n_seqs < 1 || c->max_seq_len < 1 || c->num_blocks < 1) return LRA_ERR_SHAPE;
  if (c->n_seqs > (1 << 20) || c->max_seq_len > (1 << 30)) return LRA_ERR_UNSUPPORTED;
  const int64_t room = c->block_table ? c->max_blocks_per_seq : c->num_blocks;
  if (room < 1 || room * 16 < c->max_seq_len) return LRA_ERR_SHAPE;
  if (!c->block_table && c->n_seqs != 1) return LRA_ERR_SHAPE;
  if (c->kv_head_stride < 16 * sh->head_dim || c->kv_block_stride < 16 * sh->head_dim) return LRA_ERR_SHAPE;
  if ((c->kv_head_stride | c->kv_block_stride) & 15) return LRA_ERR_SHAPE;
  if (c->kv_head_stride > (int64_t{1} << 40) || c->kv_block_stride > (int64_t{1} << 40) || c->num_blocks > (int64_t{1} << 60) / c->kv_block_stride)
    return LRA_ERR_UNSUPPORTED;
  if (c->scale_block_stride != 0 && c->scale_block_stride < sh->n_kv_heads) return LRA_ERR_SHAPE;
  if (c->scale_block_stride > (int64_t{1} << 31)) return LRA_ERR_UNSUPPORTED;
  if (c->l_row_stride < 0 || (c->l_row_stride != 0 && c->l_row_stride < sh->rank)) return LRA_ERR_SHAPE;
  if (c->l_row_stride != sh->rank && (c->l_row_stride & 7)) return LRA_ERR_SHAPE;
  if (c->l_row_stride > (int64_t{1} << 24) || (c->l_row_stride ? c->l_row_stride : sh->rank) > (int64_t{1} << 56) / c->num_blocks)
    return LRA_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) | reinterpret_cast<uintptr_t>(c->l)) & 15) return LRA_ERR_SHAPE;
  return LRA_OK;
}

lra_status check_batch8(const lra_shape* sh, const lra_cache8* c, const lra_batch* b) {
  const lra_status st = check_cache8(sh, c);
  if (st != LRA_OK) return st;
  if (!b || !b->seq_query_start || !b->query_adapter) return LRA_ERR_NULL;
  if (b->n_queries < 1 || b->max_queries_per_seq < 1 || b->max_queries_per_seq > b->n_queries) return LRA_ERR_SHAPE;
  if (b->window < 0 || b->sinks < 0) return LRA_ERR_SHAPE;
  if (static_cast<int64_t>(b->n_queries) * sh->n_q_heads > (int64_t{1} << 30)) return LRA_ERR_UNSUPPORTED;
  return LRA_OK;
}

lra_status check_new_rows(const lra_shape* sh, const lra_cache8* c, const lra_new_rows* n) {
  const lra_status st = check_cache8(sh, c);
  if (st != LRA_OK) return st;
  if (!n || !n->k || !n->v || !n->seq_start) return LRA_ERR_NULL;
  if (n->n_new < 1 || n->max_new_per_seq < 1 || n->max_new_per_seq > n->n_new) return LRA_ERR_SHAPE;
  if (!(n->rope_theta >= 0.f) || std::isinf(n->rope_theta)) return LRA_ERR_SHAPE;
  const int64_t row = static_cast<int64_t>(sh->n_kv_heads) * sh->head_dim, es = sh->dtype == LRA_BF16 ? 2 : 4;
  if (n->k_token_stride < row || n->v_token_stride < row || (n->l && n->l_token_stride < sh->rank)) return LRA_ERR_SHAPE;
  if (n->k_token_stride > (int64_t{1} << 31) || n->v_token_stride > (int64_t{1} << 31) || n->l_token_stride > (int64_t{1} << 31))
    return LRA_ERR_UNSUPPORTED;
  if (((n->k_token_stride | n->v_token_stride) * es) & 15) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(n->k) | reinterpret_cast<uintptr_t>(n->v)) & 15) return LRA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(n->l) & static_cast<uintptr_t>(es - 1)) return LRA_ERR_SHAPE;
  return LRA_OK;
}

static size_t aligned(size_t bytes) { return (bytes + 255) & ~static_cast<size_t>(255); }

static void place_states(Attn8Plan& pl, const lra_shape* sh) {
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

// The most keys that one query sees.
static int64_t keys_per_row(const lra_cache8* c, const lra_batch* b) {
  return b->window > 0 ? std::min<int64_t>(c->max_seq_len, static_cast<int64_t>(b->window) + b->sinks) : c->max_seq_len;
}

// 64 rows at most per sequence and kv head: workgroups of (kv head, key share, sequence), two to a compute unit, whose waves (four, or
// two for each of two row tiles) have a tile of 64 keys each.  More shares even out sequences of unlike lengths but leave more states:
// 16 sequences of 4 k to 64 k tokens, 28 rows, took 2, 4 and 10 % longer with four, six and eight workgroups to a compute unit.  Shares of two
// tiles to a wave: 16 rows over 8 k tokens take 14.6 us instead of 13.2.
// Of several sequences the device forms the shares by their lengths (attn8_share) where equal numbers would have 128 tiles and more, some 25 us:
// that takes 1.5 us, and rounds up a sequence's shares, so that 32 sequences of 0.5 k to 8 k tokens, two shares each, take 96 us instead of 85;
// 40 of 0.5 k to 32 k take 304 instead of 428, 100 of 0.1 k to 16 k 391 instead of 380.
static bool plan_few_rows(Attn8Plan& pl, const lra_shape* sh, const lra_cache8* c, const lra_batch* b) {
  const int64_t G = sh->n_q_heads / sh->n_kv_heads, most = b->max_queries_per_seq * G;
  if (most > 64 || c->n_seqs > 65535) return false;
  pl.row_tiles = most <= 16 ? 1 : (most <= 32 ? 2 : 4);
  const int64_t units = static_cast<int64_t>(sh->n_kv_heads) * std::min(c->n_seqs, b->n_queries);
  const int64_t chunk = b->causal ? b->max_queries_per_seq : 1;
  const int64_t key_tiles = (std::min<int64_t>(c->max_seq_len, keys_per_row(c, b) + chunk) + 63) / 64 + (b->window > 0 ? 2 : 0);
  const int64_t waves = pl.row_tiles <= 2 ? 4 : 2;
  pl.few_rows = true;
  const int64_t even = std::max<int64_t>(1, 2 * kCUs / units), per_head = std::max<int64_t>(1, 2 * kCUs / sh->n_kv_heads);
  const int64_t most_shares = std::min<int64_t>((key_tiles + waves - 1) / waves, 64);
  pl.n_splits = static_cast<int>(std::min<int64_t>(even, most_shares));
  if (c->n_seqs > 1 && c->n_seqs <= kShareSeqs && key_tiles >= 128 * even) {
    pl.n_splits = static_cast<int>(std::min<int64_t>({4 * even, per_head, most_shares}));
    pl.head_shares = static_cast<int>(per_head);
    pl.share_least = static_cast<int>(waves);
  }
  place_states(pl, sh);
  return true;
}

// A workgroup of attn8_tiles_kernel takes 128 rows of one sequence.  The key tiles of a q tile are shared where there are fewer q tiles
// than the chip has places, two per compute unit, and then so that they fill the places once; a share walks two tiles at least.  Those of
// several sequences are shared out by their lengths, on the device (attn8_tiles_per_share), into some three and a half to a unit: 12 chunks of 1 to 256
// tokens over 1 k to 8 k tokens took 179 us (170 with the wave priorities that came later), 184 in twice as many equal shares for each q tile as fill
// the places and 206 in as many; over 1 k to 32 k 395, 474 and 657; 4 of 256 over 16 k 171 and 189.  In 2.7, 4.7 and 7 to a unit the first took
// 194, 193 and 197.
// Where the q tiles need no shares, those of eight sequences and more go in the order of what they see: 32 chunks of up to 512 tokens over 0.5 k
// to 16 k (28 q heads on 4) take 799 us instead of 999, 60 of up to 128 over 1 k to 30 k 916 instead of 1041; four chunks, of which one has
// nearly all tiles, 1585 instead of 1513, and tiles in shares 2 to 10 % longer.
static bool plan_tiles(Attn8Plan& pl, const lra_shape* sh, const lra_cache8* c, const lra_batch* b) {
  const int64_t G = sh->n_q_heads / sh->n_kv_heads;
  const int64_t places = b->n_queries * G / 128 + c->n_seqs;
  if (places * sh->n_kv_heads >= (int64_t{1} << 24)) return false;  // (a grid dimension holds fewer than 2^32 threads)
  const int64_t q_tiles = std::max<int64_t>((b->n_queries * G + 127) / 128, std::min(c->n_seqs, b->n_queries));
  const int64_t chunk = b->causal ? std::min<int64_t>(b->max_queries_per_seq, 128 / G + 1) : 1;
  const int64_t key_tiles = (std::min<int64_t>(c->max_seq_len, keys_per_row(c, b) + chunk) + 63) / 64 + (b->window > 0 ? 2 : 0);
  const int64_t places_per_cu = c->n_seqs > 1 ? 4 : 2;
  pl.tiles = true;
  pl.tile_places = static_cast<int>(places);
  pl.n_splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({places_per_cu * kCUs / (q_tiles * sh->n_kv_heads), (key_tiles + 1) / 2, 64})));
  if (pl.n_splits > 1 && c->n_seqs > 1 && c->n_seqs <= kShareSeqs) {
    pl.head_shares = std::max(1, 7 * kCUs / 2 / sh->n_kv_heads);
    pl.n_splits = static_cast<int>(std::min<int64_t>({(3 * pl.n_splits + 1) / 2, (key_tiles + 1) / 2, 64}));
  }
  pl.longest_first = pl.n_splits == 1 && c->n_seqs >= 8 && c->n_seqs <= kShareSeqs;
  // states also where the rows of a tile have adapters of their own (the merge kernel applies B_V row by row), and at d = 128 and ranks
  // above 32 (with the product by B_V behind its loop the kernel goes to scratch memory)
  if (pl.n_splits > 1 || !b->causal || (sh->head_dim == 128 && sh->rank > 32)) place_states(pl, sh);
  return true;
}

Attn8Plan plan_attn8(const lra_shape* sh, const lra_cache8* c, const lra_batch* b, const Tuning& tune) {
  Attn8Plan pl{};
  const int64_t rows = static_cast<int64_t>(b->n_queries) * sh->n_q_heads, keys = keys_per_row(c, b);
  pl.rows = static_cast<int>(rows);
  pl.launchable = true;
  if (sh->dtype == LRA_BF16 && sh->rank % 8 == 0 && tune.variant != 1) {
    if (tune.variant == 0 && plan_few_rows(pl, sh, c, b)) return pl;
    if (plan_tiles(pl, sh, c, b)) return pl;
  }
  // vector-ALU kernel: one workgroup per row and share, three to a compute unit; a share of 128 keys at least (a window of 256 keys
  // and 16 rows take 10.2 us, 2 more in shares of 256)
  pl.n_splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({3 * kCUs / rows, (keys + 127) / 128, 64})));
  pl.launchable = rows < (int64_t{1} << 24);  // (a grid dimension holds fewer than 2^32 threads)
  if (pl.launchable) place_states(pl, sh);
  return pl;
}

}  // namespace lra
