// Parameters of the kernels behind lra_key_weights.
#pragma once

#include "lra_batch.h"

namespace lra {

struct WeightsParams : BatchParams {
  // vector-ALU kernels: Qt [rows][rank], lse [rows], row = query Hq + q head.  MFMA kernels: Qt as bf16 (below), lse
  // [Hkv][row], row = query group + q head of the group.  lse: base-2 logarithm of the row's sum, +inf (MFMA) or -inf where it
  // sees nothing.
  float* qt;
  float* lse;
  float* stats;    // MFMA: [Hkv][shares][row][2], maximum and sum of a key share's scores, base 2
  float* weights;  // [n_seqs][weights_stride]
  int64_t weights_stride;
  float decay;
  int32_t rows_per_head;  // n_queries x group
  int32_t sum_tiles;      // weights_sum_rows_kernel: tiles of 32 keys per workgroup
};

hipError_t launch_key_weights_mfma(const WeightsParams& p, hipStream_t s);

}  // namespace lra
