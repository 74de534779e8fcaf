// Tiles of a gradient's terms, with the weights as the layer has them.
#include "bq_linear_tile.h"

namespace bq {

template <int kWBits>
static hipError_t launch(const LinearArgs &A, int terms, LinearTile tile, hipStream_t stream)
{
    if (terms == 3)
        return tile == kTileLarge ? launch_tile<16, kWBits, 3, TileLarge3, true>(A, stream) : launch_tile<16, kWBits, 3, TileDeep3, true>(A, stream);
    if (tile == kTileLarge) return launch_tile<16, kWBits, 2, TileLarge, true>(A, stream);
    if (tile == kTileTall) return launch_tile<16, kWBits, 2, TileTall, true>(A, stream);
    if (tile == kTileMiddle) return launch_tile<16, kWBits, 2, TileMiddle, true>(A, stream);
    if constexpr (kWBits == 8) {
        if (tile == kTileDeep) return launch_tile<16, 8, 2, TileDeep, true>(A, stream);
    }
    return launch_tile<16, kWBits, 2, TileSmall, true>(A, stream);
}

hipError_t launch_linear_tile_across(const LinearArgs &A, int wbits, int terms, LinearTile tile, hipStream_t stream)
{
    if (wbits == 8) return launch<8>(A, terms, tile, stream);
    if (wbits == 4) return launch<4>(A, terms, tile, stream);
    return launch<2>(A, terms, tile, stream);
}

}  // namespace bq
