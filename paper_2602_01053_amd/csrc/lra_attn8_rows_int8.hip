// Instantiations of the few-rows kernels over LRA_INT8 codes (a file each: they compile side by side).
#include "lra_attn8_rows32.h"

namespace lra {

hipError_t launch_attn8_rows_int8(const Batch8Params& p, int row_tiles, hipStream_t s) {
  return p.head_dim == 128 ? launch_attn8_rows<128, LRA_INT8>(p, row_tiles, s) : launch_attn8_rows<64, LRA_INT8>(p, row_tiles, s);
}

}  // namespace lra
