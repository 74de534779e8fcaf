// Eight neighbouring entries of a row that starts anywhere and ends anywhere.  Memory takes a load of 16 bytes at any address, so such
// rows cost their extra lines and the last piece's single entries, not a path of their own.
#pragma once

#include "bq_cascade.h"

namespace bq {

template <typename T>
__device__ __forceinline__ Raw8 load_whole_piece(const T *p)
{
    Raw8 r;
    __builtin_memcpy(&r.lo, p, 16);
    if (sizeof(T) == 4) __builtin_memcpy(&r.hi, (const char *)p + 16, 16);
    return r;
}

// entries p[0 .. 7], of which `left` are the row's; the others are 0 and not read.
template <typename T>
__device__ __forceinline__ Raw8 load_piece(const T *p, int left)
{
    if (left >= 8) return load_whole_piece(p);
    Raw8 r;
    uint32_t w[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= left) continue;
        if (sizeof(T) == 4)
            w[i] = ((const uint32_t *)p)[i];
        else
            w[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << (16 * (i % 2));
    }
    r.lo = make_uint4(w[0], w[1], w[2], w[3]);
    if (sizeof(T) == 4) r.hi = make_uint4(w[4], w[5], w[6], w[7]);
    return r;
}

// eight bytes, of which `left` are the row's
__device__ __forceinline__ void store_piece(int8_t *p, uint2 v, int left)
{
    if (left >= 8) {
        __builtin_memcpy(p, &v, 8);
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) p[i] = (int8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
}

}  // namespace bq
