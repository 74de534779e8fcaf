// Which kernel takes a product of codes.
#include "bq_linear.h"

namespace bq {

namespace {

constexpr int kCUs = 256;

bool fast_layout(const LinearArgs &A, int xbits, int wbits)
{
    const int64_t x_bytes = (int64_t)A.k * xbits / 8, w_bytes = (int64_t)A.k * wbits / 8;
    // whole 16-byte pieces of both operands; offsets within a tile of 256 rows in 32 bits
    return (uintptr_t)A.x % 16 == 0 && (uintptr_t)A.w % 16 == 0 && A.ldx % 16 == 0 && A.ldw % 16 == 0 && A.k * xbits % 128 == 0 &&
           A.k * wbits % 128 == 0 && x_bytes > 0 && w_bytes > 0 && A.ldx < (int64_t)1 << 23 && A.ldw < (int64_t)1 << 23;
}

}  // namespace

hipError_t launch_linear(const LinearArgs &A0, int xbits, int wbits, int planes, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor /= (float)((1 << (8 - xbits)) * (1 << (8 - wbits)));
    const size_t size = A.dtype == BQ_F32 ? 4 : 2;
    A.y_quads = (uintptr_t)A.y % 16 == 0 && A.ldy * size % 16 == 0;
    if (!fast_layout(A, xbits, wbits)) return launch_linear_any(A, xbits, wbits, planes, stream);
    const int64_t each = (A.rows + A.experts - 1) / A.experts;  // rows of an expert, if they are spread evenly
    if (each <= 64 / (planes == 1 ? 1 : 2)) {
        const int blocks = each <= 16 ? 1 : each <= 32 ? 2 : 4;
        if (xbits == 8) return launch_linear_rows8(A, wbits, planes, blocks, stream);
        return launch_linear_rows4(A, wbits, blocks, stream);
    }
    const int64_t tokens = planes == 1 ? 256 : 128, channels = planes == 3 ? 128 : 256;
    const int64_t large_tiles = ((each + tokens - 1) / tokens) * A.experts * ((A.n + channels - 1) / channels);
    const bool large = large_tiles >= kCUs;
    if (planes > 1) return launch_linear_tile_digits(A, planes, large, stream);
    if (xbits == 8) return launch_linear_tile8(A, wbits, large, stream);
    return launch_linear_tile4(A, wbits, large, stream);
}

}  // namespace bq
