// The kernels of ffn_s4_tiled.h for groups of 256 numbers.
#include "ffn_s4_tiled.h"

namespace icnn {

hipError_t launch_tiled_s4_256(const LinearS4Args &a, int tile, hipStream_t st) { return launch_s4_tiles<256>(a, tile, st); }

}  // namespace icnn
