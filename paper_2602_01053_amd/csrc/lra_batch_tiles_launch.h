// Choice among the instantiations of the batch's tile-walking kernel.
#pragma once

#include "lra_batch_tiles.h"

namespace lra {

// Forms that few calls take (a rotated key side, pools beyond 32-bit byte offsets) leave states for the merge kernel whatever
// the number of shares: half the instantiations.
template <int D, int RP, bool PAGED, bool POOL, bool SPLIT_ONLY>
static hipError_t launch_batch_tiles_bk(const BatchParams& p, dim3 grid, hipStream_t s) {
  const bool has_bk = p.b_k != nullptr;
  if (p.part_ml == nullptr) {
    if constexpr (SPLIT_ONLY) return hipErrorInvalidValue;
    else if (has_bk) hipLaunchKernelGGL((batch_tiles_kernel<D, RP, PAGED, POOL, true, false, false>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((batch_tiles_kernel<D, RP, PAGED, POOL, false, false, false>), grid, dim3(256), 0, s, p);
  } else if (has_bk) {
    hipLaunchKernelGGL((batch_tiles_kernel<D, RP, PAGED, POOL, true, true, false>), grid, dim3(256), 0, s, p);
  } else {
    hipLaunchKernelGGL((batch_tiles_kernel<D, RP, PAGED, POOL, false, true, false>), grid, dim3(256), 0, s, p);
  }
  return hipGetLastError();
}

template <int D, int RP>
static hipError_t launch_batch_tiles_rp(const BatchParams& p, dim3 grid, hipStream_t s) {
  const bool paged = p.block_size != 0;
  const bool pool = paged && prefill_pool_fits(p);
  if (p.b_k != nullptr && p.key_rope_theta > 0.f) {
    if (p.part_ml == nullptr) return hipErrorInvalidValue;
    if (pool) hipLaunchKernelGGL((batch_tiles_kernel<D, RP, true, true, false, true, true>), grid, dim3(256), 0, s, p);
    else if (paged) hipLaunchKernelGGL((batch_tiles_kernel<D, RP, true, false, false, true, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((batch_tiles_kernel<D, RP, false, false, false, true, true>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
  }
  if (pool) return launch_batch_tiles_bk<D, RP, true, true, false>(p, grid, s);
  if (paged) return launch_batch_tiles_bk<D, RP, true, false, true>(p, grid, s);
  return launch_batch_tiles_bk<D, RP, false, false, false>(p, grid, s);
}

template <int D>
static hipError_t launch_batch_tiles(const BatchParams& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.tile_places * p.n_kv_heads), p.n_splits);
  if (p.rank <= 16) return launch_batch_tiles_rp<D, 16>(p, grid, s);
  if (p.rank <= 32) return launch_batch_tiles_rp<D, 32>(p, grid, s);
  return launch_batch_tiles_rp<D, 64>(p, grid, s);
}

}  // namespace lra
