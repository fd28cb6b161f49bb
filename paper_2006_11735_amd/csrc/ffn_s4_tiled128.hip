// The kernels of ffn_s4_tiled.h for groups of 128 numbers.
#include "ffn_s4_tiled.h"

namespace icnn {

hipError_t launch_tiled_s4_128(const LinearS4Args &a, int tile, hipStream_t st) { return launch_s4_tiles<128>(a, tile, st); }

}  // namespace icnn
