// Tiles of a gradient's digits, with the weights as the layer has them.
#include "bq_linear_tile.h"

namespace bq {

template <int kWBits>
static hipError_t launch(const LinearArgs &A, int planes, LinearTile tile, hipStream_t stream)
{
    if (planes == 3)
        return tile == kTileLarge ? launch_tile<8, kWBits, 3, TileLarge3, true>(A, stream) : launch_tile<8, kWBits, 3, TileDeep3, true>(A, stream);
    if (tile == kTileLarge) return launch_tile<8, kWBits, 2, TileLarge, true>(A, stream);
    if (tile == kTileTall) return launch_tile<8, kWBits, 2, TileTall, true>(A, stream);
    if (tile == kTileMiddle) return launch_tile<8, kWBits, 2, TileMiddle, true>(A, stream);
    if constexpr (kWBits == 8) {
        if (tile == kTileDeep) return launch_tile<8, 8, 2, TileDeep, true>(A, stream);
    }
    return launch_tile<8, kWBits, 2, TileSmall, true>(A, stream);
}

hipError_t launch_linear_tile_across(const LinearArgs &A, int wbits, int planes, LinearTile tile, hipStream_t stream)
{
    if (wbits == 8) return launch<8>(A, planes, tile, stream);
    if (wbits == 4) return launch<4>(A, planes, tile, stream);
    return launch<2>(A, planes, tile, stream);
}

}  // namespace bq
