// Tiles of float32 products (see tile.h).
#include "tile_launch.h"

namespace hr {
template hipError_t launch_tiles<float, false>(const Tiling&, const TilePair&, int, hipStream_t);
template hipError_t launch_tiles<float, true>(const Tiling&, const TilePair&, int, hipStream_t);
}  // namespace hr
