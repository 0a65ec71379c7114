// Attention of a batch with a window and sinks: entry points.
// Declarations and argument contracts are in lra_attn.h.
#include "lra_batch.h"

#include <cmath>

#include "lra_attn.h"
#include "lra_batch_plan.h"

namespace lra {

BatchParams batch_params(const lra_shape* sh, const lra_cache* c, const lra_adapters* ad, const lra_batch* b, const void* q) {
  BatchParams p{};
  p.q = q;
  p.k_base = c->k_base;
  p.v_base = c->v_base;
  p.l = c->l;
  p.b_k = ad->b_k;
  p.b_v = ad->b_v;
  p.n_adapters = ad->n_adapters;
  p.block_table = c->block_table;
  p.seq_lens = c->seq_lens;
  p.query_adapter = b->query_adapter;
  p.seq_query_start = b->seq_query_start;
  p.kv_token_stride = c->kv_token_stride;
  p.kv_head_stride = c->kv_head_stride;
  p.kv_block_stride = c->kv_block_stride;
  p.l_row_stride = c->l_row_stride ? c->l_row_stride : sh->rank;
  p.l_adapter_stride = c->l_adapter_stride;
  p.n_q_heads = sh->n_q_heads;
  p.n_kv_heads = sh->n_kv_heads;
  p.group = sh->n_q_heads / sh->n_kv_heads;
  p.head_dim = sh->head_dim;
  p.rank = sh->rank;
  p.block_size = c->block_size;
  p.max_blocks_per_seq = c->max_blocks_per_seq;
  p.num_blocks = c->num_blocks;
  p.n_seqs = c->n_seqs;
  p.max_seq_len = c->max_seq_len;
  p.n_queries = b->n_queries;
  p.max_queries_per_seq = b->max_queries_per_seq;
  p.n_new = 1;
  p.scale = sh->scale > 0.f ? sh->scale : 1.0f / std::sqrt(static_cast<float>(sh->head_dim));
  p.key_rope_theta = sh->key_rope_theta;
  p.causal = b->causal != 0;
  // (longer ones change nothing, and sums with positions stay in 32 bits)
  p.window = b->window < c->max_seq_len ? b->window : c->max_seq_len;
  p.sinks = b->window <= 0 ? 0 : (b->sinks < c->max_seq_len ? b->sinks : c->max_seq_len);
  return p;
}

}  // namespace lra

using namespace lra;

extern "C" {

size_t lra_batch_workspace_bytes(const lra_shape* shape, const lra_cache* cache, const lra_batch* batch, const lra_tuning* tuning) {
  if (check_batch(shape, cache, batch) != LRA_OK) return static_cast<size_t>(-1);
  return batch_workspace_bytes(shape, cache, batch, resolve_tuning(tuning));
}

lra_status lra_attn_batch(const lra_shape* shape, const lra_cache* cache, const lra_adapters* adapters, const lra_batch* batch,
                          const void* q, void* out, void* workspace, size_t workspace_bytes, const lra_tuning* tuning, void* stream) {
  const lra_status st = check_batch(shape, cache, batch);
  if (st != LRA_OK) return st;
  if (!adapters || !q || !out) return LRA_ERR_NULL;
  if (adapters->n_adapters < 1) return LRA_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(adapters->b_k) |
       reinterpret_cast<uintptr_t>(adapters->b_v)) & 15)
    return LRA_ERR_SHAPE;
  const BatchPlan pl = plan_batch(shape, cache, batch, resolve_tuning(tuning), adapters->b_k != nullptr);
  if (!pl.launchable) return LRA_ERR_UNSUPPORTED;
  if (pl.bytes > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < pl.bytes)) return LRA_ERR_WORKSPACE;
  BatchParams p = batch_params(shape, cache, adapters, batch, q);
  p.out = out;
  p.split_keys = pl.split_keys;
  p.n_splits = pl.n_splits;
  if (pl.states) {
    char* ws = static_cast<char*>(workspace);
    p.part_ml = reinterpret_cast<float*>(ws + pl.off_ml);
    p.part_o = reinterpret_cast<float*>(ws + pl.off_o);
    p.part_lr = reinterpret_cast<float*>(ws + pl.off_lr);
    p.part_adapter = reinterpret_cast<int32_t*>(ws + pl.off_adapter);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = shape->dtype == LRA_BF16;
  if (pl.few_rows) {
    if (launch_batch_rows(p, s) != hipSuccess) return LRA_ERR_HIP;
  } else if (pl.tiles) {
    p.row_mul = (65535 + p.group) / p.group;
    p.tile_places = pl.tile_places;
    p.tile_per_query = pl.tile_per_query;
    if ((p.head_dim == 128 ? launch_batch_tiles_d128(p, s) : launch_batch_tiles_d64(p, s)) != hipSuccess) return LRA_ERR_HIP;
  } else if (launch_batch_partials(p, bf16, pl.rows, s) != hipSuccess) {
    return LRA_ERR_HIP;
  }
  if (pl.states && launch_merge(p, bf16, pl.rows, s) != hipSuccess) return LRA_ERR_HIP;
  return LRA_OK;
}

}  // extern "C"
