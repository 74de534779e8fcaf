// Tiles of 4-bit codes.
#include "bq_linear_tile.h"

namespace bq {

hipError_t launch_linear_tile4(const LinearArgs &A, int wbits, bool large, hipStream_t stream)
{
    if (wbits == 8) return large ? launch_tile<4, 8, 1, TileLarge>(A, stream) : launch_tile<4, 8, 1, TileSmall>(A, stream);
    if (wbits == 4) return large ? launch_tile<4, 4, 1, TileLarge>(A, stream) : launch_tile<4, 4, 1, TileSmall>(A, stream);
    return large ? launch_tile<4, 2, 1, TileLarge>(A, stream) : launch_tile<4, 2, 1, TileSmall>(A, stream);
}

}  // namespace bq
