// Few rows of a gradient's terms.
#include "bq_linear_rows.h"

namespace bq {

hipError_t launch_linear_rows_terms(const LinearArgs &A, int terms, int blocks, int cols, hipStream_t stream)
{
    if (terms == 2) return launch_rows_of<16, 8, 2>(A, blocks, cols, stream);
    return launch_rows_of<16, 8, 3>(A, blocks, cols, stream);
}

}  // namespace bq
