// Instantiations of the tile-walking kernel over LRA_INT8 codes (a file each: they compile side by side).
#include "lra_attn8_tiles.h"

namespace lra {

hipError_t launch_attn8_tiles_int8(const Batch8Params& p, hipStream_t s) {
  return p.head_dim == 128 ? launch_attn8_tiles<128, LRA_INT8>(p, s) : launch_attn8_tiles<64, LRA_INT8>(p, s);
}

}  // namespace lra
