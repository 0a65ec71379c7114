// Instantiations of the batch's tile-walking kernel for head dimension 128 (a file each: they compile side by side).
#include "lra_batch_tiles_launch.h"

namespace lra {

hipError_t launch_batch_tiles_d128(const BatchParams& p, hipStream_t s) { return launch_batch_tiles<128>(p, s); }

}  // namespace lra
