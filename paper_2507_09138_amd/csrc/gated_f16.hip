// Tiles of float16 products (see tile.h).
#include "tile_launch.h"

namespace hr {
template hipError_t launch_tiles<_Float16, false>(const Tiling&, const TilePair&, int, hipStream_t);
template hipError_t launch_tiles<_Float16, true>(const Tiling&, const TilePair&, int, hipStream_t);
}  // namespace hr
