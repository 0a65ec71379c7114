// Parameters of the kernels behind lra_key_weights.
#pragma once

#include "lra_batch.h"

namespace lra {

struct WeightsParams : BatchParams {
  // vector-ALU kernels: Qt [rows][rank], statistics [rows][shares][2], row = query Hq + q head.  MFMA kernels: Qt as bf16
  // (weights_stats_mfma_kernel), statistics [Hkv][shares][row][2] and lse [Hkv][row], row = query group + q head of the group; lse
  // the base-2 logarithm of the row's sum, +inf where it sees nothing.  Statistics: maximum and sum of a share's scores, base 2.
  float* qt;
  float* lse;
  float* stats;
  float* weights;  // [n_seqs][weights_stride]
  int64_t weights_stride;
  float decay;
  int32_t rows_per_head;  // n_queries x group
  int32_t sum_tiles;      // weights_sum_rows_kernel: tiles of 32 keys per workgroup
  int32_t sum_groups;     // weights_sum_mfma_kernel: groups that the kv heads are divided into
  float* group_sums;      // [sum_groups][n_seqs][max_seq_len], more than one group only
};

hipError_t launch_key_weights_mfma(const WeightsParams& p, hipStream_t s);

}  // namespace lra
