// Tiles of a gradient's digits.
#include "bq_linear_tile.h"

namespace bq {

hipError_t launch_linear_tile_digits(const LinearArgs &A, int planes, bool large, hipStream_t stream)
{
    if (planes == 2) return large ? launch_tile<8, 8, 2, TileLarge>(A, stream) : launch_tile<8, 8, 2, TileSmall>(A, stream);
    return large ? launch_tile<8, 8, 3, TileLarge3>(A, stream) : launch_tile<8, 8, 3, TileSmall3>(A, stream);
}

}  // namespace bq
