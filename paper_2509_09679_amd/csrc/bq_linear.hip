// Which kernel takes a product of codes.
#include "bq_linear.h"

namespace bq {

hipError_t launch_linear(const LinearArgs &A0, int xbits, int wbits, int planes, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor = 1.0f / (float)((1 << (8 - xbits)) * (1 << (8 - wbits)));
    return launch_linear_any(A, xbits, wbits, planes, stream);
}

}  // namespace bq
