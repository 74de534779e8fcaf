// Few rows of 8-bit codes.
#include "bq_linear_rows.h"

namespace bq {

hipError_t launch_linear_rows8(const LinearArgs &A, int wbits, int blocks, int cols, hipStream_t stream)
{
    if (wbits == 8) return launch_rows_of<8, 8, 1>(A, blocks, cols, stream);
    if (wbits == 4) return launch_rows_of<8, 4, 1>(A, blocks, cols, stream);
    return launch_rows_of<8, 2, 1>(A, blocks, cols, stream);
}

}  // namespace bq
