// int8 tile GEMM instances: 128x128, 128x64 and 64x64 tiles. The kernel is in gemm_tile.h.
#include "gemm_tile.h"

namespace ps {
PS_I8_INSTANCES_SMALL(PS_I8_INSTANTIATE)
}  // namespace ps
