// Few rows of 4-bit codes.
#include "bq_linear_rows.h"

namespace bq {

hipError_t launch_linear_rows4(const LinearArgs &A, int wbits, int blocks, int cols, hipStream_t stream)
{
    if (wbits == 8) return launch_rows_of<4, 8, 1>(A, blocks, cols, stream);
    if (wbits == 4) return launch_rows_of<4, 4, 1>(A, blocks, cols, stream);
    return launch_rows_of<4, 2, 1>(A, blocks, cols, stream);
}

}  // namespace bq
