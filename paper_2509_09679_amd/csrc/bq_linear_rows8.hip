// Few rows of 8-bit codes, and of a gradient's digits.
#include "bq_linear_rows.h"

namespace bq {

hipError_t launch_linear_rows8(const LinearArgs &A, int wbits, int planes, int blocks, int cols, hipStream_t stream)
{
    if (planes == 2) return launch_rows_of<8, 8, 2>(A, blocks, cols, stream);
    if (planes == 3) return launch_rows_of<8, 8, 3>(A, blocks, cols, stream);
    if (wbits == 8) return launch_rows_of<8, 8, 1>(A, blocks, cols, stream);
    if (wbits == 4) return launch_rows_of<8, 4, 1>(A, blocks, cols, stream);
    return launch_rows_of<8, 2, 1>(A, blocks, cols, stream);
}

}  // namespace bq
