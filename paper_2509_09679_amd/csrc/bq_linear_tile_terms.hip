// Tiles of a gradient's terms.
#include "bq_linear_tile.h"

namespace bq {

hipError_t launch_linear_tile_terms(const LinearArgs &A, int terms, LinearTile tile, hipStream_t stream)
{
    if (terms == 3) return tile == kTileLarge ? launch_tile<16, 8, 3, TileLarge3>(A, stream) : launch_tile<16, 8, 3, TileDeep3>(A, stream);
    if (tile == kTileLarge) return launch_tile<16, 8, 2, TileLarge>(A, stream);
    if (tile == kTileTall) return launch_tile<16, 8, 2, TileTall>(A, stream);
    if (tile == kTileMiddle) return launch_tile<16, 8, 2, TileMiddle>(A, stream);
    if (tile == kTileDeep) return launch_tile<16, 8, 2, TileDeep>(A, stream);
    return launch_tile<16, 8, 2, TileSmall>(A, stream);
}

}  // namespace bq
