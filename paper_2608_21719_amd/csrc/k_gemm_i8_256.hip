// int8 tile GEMM instances: 256x256 tiles. The kernel is in gemm_tile.h.
#include "gemm_tile.h"

namespace ps {
PS_I8_INSTANCES_256(PS_I8_INSTANTIATE)
}  // namespace ps
