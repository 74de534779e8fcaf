// Tiles of 4-bit codes.
#include "bq_linear_tile.h"

namespace bq {

template <int kWBits>
static hipError_t launch(const LinearArgs &A, LinearTile tile, hipStream_t stream)
{
    if (tile == kTileLarge) return launch_tile<4, kWBits, 1, TileLarge>(A, stream);
    if (tile == kTileMiddle) return launch_tile<4, kWBits, 1, TileMiddle>(A, stream);
    if constexpr (kWBits == 8) {
        if (tile == kTileDeep) return launch_tile<4, 8, 1, TileDeep>(A, stream);
    }
    return launch_tile<4, kWBits, 1, TileSmall>(A, stream);
}

hipError_t launch_linear_tile4(const LinearArgs &A, int wbits, LinearTile tile, hipStream_t stream)
{
    if (wbits == 8) return launch<8>(A, tile, stream);
    if (wbits == 4) return launch<4>(A, tile, stream);
    return launch<2>(A, tile, stream);
}

}  // namespace bq
