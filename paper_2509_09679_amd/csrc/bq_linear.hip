// The launch of a product of codes or a gradient: the kernel that bq_linear_choice.h chooses.
#include "bq_linear.h"

namespace bq {

namespace {

bool fast_layout(const LinearArgs &A, int xbits, int wbits)
{
    // whole 16-byte pieces of both operands; offsets within a tile of 256 rows in 32 bits
    return (uintptr_t)A.x % 16 == 0 && (uintptr_t)A.w % 16 == 0 && A.ldx % 16 == 0 && A.ldw % 16 == 0 && A.k * (int64_t)xbits % 128 == 0 &&
           A.k * (int64_t)wbits % 128 == 0 && A.ldx < (int64_t)1 << 23 && A.ldw < (int64_t)1 << 23;
}

}  // namespace

hipError_t launch_linear(const LinearArgs &A0, int xbits, int wbits, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor /= (float)((1 << (8 - xbits)) * (1 << (8 - wbits)));
    if (!fast_layout(A, xbits, wbits)) return launch_linear_any(A, xbits, wbits, stream);
    const LinearChoice c = choose_codes(size_of(A), xbits, wbits);
    if (c.few) {
        if (xbits == 4) return launch_linear_rows4(A, wbits, c.blocks, c.cols, stream);
        return launch_linear_rows8(A, wbits, c.blocks, c.cols, stream);
    }
    if (xbits == 8) return launch_linear_tile8(A, wbits, c.tile, stream);
    return launch_linear_tile4(A, wbits, c.tile, stream);
}

hipError_t launch_linear_terms(const LinearArgs &A, int terms, hipStream_t stream)
{
    const LinearChoice c = choose_terms(size_of(A), 8, terms, false);
    return c.few ? launch_linear_rows_terms(A, terms, c.blocks, c.cols, stream) : launch_linear_tile_terms(A, terms, c.tile, stream);
}

bool linear_across_is_quicker(const LinearArgs &A, int wbits, int terms)
{
    if ((uintptr_t)A.w % 16 != 0 || A.ldw % 16 != 0 || A.n * (int64_t)wbits % 128 != 0 || A.ldw >= (int64_t)1 << 23) return false;
    return across_is_quicker(size_of(A), wbits, terms);
}

hipError_t launch_linear_across(const LinearArgs &A, int wbits, int terms, hipStream_t stream)
{
    return launch_linear_tile_across(A, wbits, terms, choose_terms(size_of(A), wbits, terms, true).tile, stream);
}

}  // namespace bq
