// int8 tile GEMM instances: 192x256 and 128x256 tiles. The kernel is in gemm_tile.h.
#include "gemm_tile.h"

namespace ps {
PS_I8_INSTANCES_WIDE(PS_I8_INSTANTIATE)
}  // namespace ps
