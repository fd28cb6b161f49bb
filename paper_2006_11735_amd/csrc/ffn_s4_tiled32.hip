// The kernels of ffn_s4_tiled.h for groups of 32 numbers.
#include "ffn_s4_tiled.h"

namespace icnn {

hipError_t launch_tiled_s4_32(const LinearS4Args &a, int tile, hipStream_t st) { return launch_s4_tiles<32>(a, tile, st); }

}  // namespace icnn
