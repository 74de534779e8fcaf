// Codes as the matrix cores take them: 16 bytes per lane, from 16 codes of 8, 4 or 2 bits.
#pragma once

#include "bq_linear.h"

namespace bq {

// 8 codes of 4 bits, as bytes that hold 16 times the code.  Natural order costs a byte interleave; where both operands have 4 bits
// they can stay in the order (even codes, odd codes), which the sum does not see.
template <bool kNatural>
__device__ __forceinline__ void unpack4bit(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    const uint32_t even = (w << 4) & 0xF0F0F0F0u, odd = w & 0xF0F0F0F0u;
    if (kNatural) {
        lo = __builtin_amdgcn_perm(odd, even, 0x05010400u);
        hi = __builtin_amdgcn_perm(odd, even, 0x07030602u);
    } else {
        lo = even;
        hi = odd;
    }
}

// 16 codes of 2 bits, as bytes that hold 64 times the code, in natural order
__device__ __forceinline__ i32x4 unpack2bit(uint32_t w)
{
    const uint32_t t0 = (w << 6) & 0xC0C0C0C0u, t1 = (w << 4) & 0xC0C0C0C0u, t2 = (w << 2) & 0xC0C0C0C0u, t3 = w & 0xC0C0C0C0u;
    const uint32_t a = __builtin_amdgcn_perm(t1, t0, 0x05010400u), b = __builtin_amdgcn_perm(t3, t2, 0x05010400u);
    const uint32_t c = __builtin_amdgcn_perm(t1, t0, 0x07030602u), d = __builtin_amdgcn_perm(t3, t2, 0x07030602u);
    i32x4 r;
    r[0] = (int)__builtin_amdgcn_perm(b, a, 0x05040100u);
    r[1] = (int)__builtin_amdgcn_perm(b, a, 0x07060302u);
    r[2] = (int)__builtin_amdgcn_perm(d, c, 0x05040100u);
    r[3] = (int)__builtin_amdgcn_perm(d, c, 0x07060302u);
    return r;
}

// the 16 codes of step s out of a lane's packed words (8 bits: 4 words per step; 4 bits: 2; 2 bits: 1)
template <int kBits, bool kNatural, int kWords>
__device__ __forceinline__ i32x4 step_codes(const uint32_t (&w)[kWords], int s)
{
    i32x4 r;
    if constexpr (kBits == 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = (int)w[4 * s + j];
    } else if constexpr (kBits == 4) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t lo, hi;
            unpack4bit<kNatural>(w[2 * s + j], lo, hi);
            r[2 * j] = (int)lo;
            r[2 * j + 1] = (int)hi;
        }
    } else {
        r = unpack2bit(w[s]);
    }
    return r;
}

// One wave instruction: 16 bytes per lane from base + offset into LDS, in lane order.  The compiler does not see it: the reader waits
// for vmcnt itself, and for its own reads before their place is loaded again.  (m0 is reserved: the compiler sets it where it needs it, and
// naming it as clobbered gives a warning and the same code.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, const uint8_t *base)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" : : "v"(offset), "s"(lds), "s"(base) : "memory");
}

// Where the 16-byte pieces of LDS rows of kRowBytes lie: piece p of a row at p ^ lds_turn(row), so that reads find their banks free.  A
// read of 16 bytes per lane goes 16 lanes at a time, {0-3, 12-15, 20-27} and {4-11, 16-19, 28-31} of either half of the wave (measured:
// two lanes that read the same banks cost a cycle exactly if both are in one of these sets), over 64 banks: 256 bytes, 2 or 4
// rows.  For reads where lane i + 16 g takes piece kPieces g + .. of row i.
template <int kRowBytes, int kPieces>
__device__ __forceinline__ int lds_turn(int row)
{
    static_assert((kRowBytes == 128 && (kPieces == 2 || kPieces == 4)) || (kRowBytes == 64 && kPieces == 1), "the turns worked out");
    return kRowBytes == 64 ? (row >> 2) & 2 : ((row >> 1) & 1) | (kPieces == 2 ? (row >> 1) & 4 : (row >> 2) & 2);
}

// ---- codes of weights as binary16 numbers, for a gradient.  A field in the low bits of a binary16 number with the exponent of 1024 is 1024
// plus its value; packed binary16 operations move that to the code itself, exactly.

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t f16_pair(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// the fields of kBits at bit kAt of both halves of w, as codes: one instruction picks them, turns their top bits round and sets the exponent
template <int kBits, int kAt>
__device__ __forceinline__ uint32_t half_fields(uint32_t w)
{
    constexpr uint32_t kMask = ((1u << kBits) - 1) << kAt, kTurn = 0x6400u | 1u << (kAt + kBits - 1);
    constexpr float kStep = 1.0f / (1 << kAt), kOffset = -(1024.0f * kStep + (1 << (kBits - 1)));
    const f16x2 v = __builtin_bit_cast(f16x2, __builtin_amdgcn_bitop3_b32(w, kMask << 16 | kMask, kTurn << 16 | kTurn, 0x6A));  // (w & mask) ^ turn
    return f16_pair(__builtin_elementwise_fma(v, f16x2{(_Float16)kStep, (_Float16)kStep}, f16x2{(_Float16)kOffset, (_Float16)kOffset}));
}

// 8 codes of 8 bits, in order
__device__ __forceinline__ i32x4 half_codes8(uint32_t lo, uint32_t hi)
{
    i32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = __builtin_amdgcn_perm(0x64646464u, (j < 2 ? lo : hi) ^ 0x80808080u, j % 2 ? 0x04030402u : 0x04010400u);
        r[j] = (int)f16_pair(__builtin_bit_cast(f16x2, w) - f16x2{(_Float16)1152.0f, (_Float16)1152.0f});
    }
    return r;
}

// 8 codes of 4 bits, as 0, 4, 1, 5, 2, 6, 3, 7
__device__ __forceinline__ i32x4 half_codes4(uint32_t w)
{
    const uint32_t v = w >> 8;
    return i32x4{(int)half_fields<4, 0>(w), (int)half_fields<4, 4>(w), (int)half_fields<4, 0>(v), (int)half_fields<4, 4>(v)};
}

// the same of the even channel (odd = 0) or the odd one of 8 fields of 4 bits that hold two codes of 2 bits each
__device__ __forceinline__ i32x4 half_codes2(uint32_t w, int odd)
{
    const uint32_t v = w >> 8;
    if (odd) return i32x4{(int)half_fields<2, 2>(w), (int)half_fields<2, 6>(w), (int)half_fields<2, 2>(v), (int)half_fields<2, 6>(v)};
    return i32x4{(int)half_fields<2, 0>(w), (int)half_fields<2, 4>(w), (int)half_fields<2, 0>(v), (int)half_fields<2, 4>(v)};
}

// ---- what products of codes (int32 sums) and gradients (binary16 terms, float32 sums) have in common

template <bool kFloat>
struct SumType {
    typedef i32x4 type;
};
template <>
struct SumType<true> {
    typedef f32x4 type;
};

__device__ __forceinline__ i32x4 multiply(i32x4 w, i32x4 x, i32x4 sum) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, sum, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(i32x4 w, i32x4 x, f32x4 sum)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), sum, 0, 0, 0);
}

// The value of one result.  The fields' factor, a power of two, goes to the sum, where it is exact: a scale near float32's smallest would
// lose digits to it.
__device__ __forceinline__ float scaled(int sum, float fields, float xs, float ws) { return (float)sum * fields * xs * ws; }

// a gradient's: the terms behind the first are kept 2^11 times their size (bq_linear_bwd.hip)
constexpr float kLowerTerms = 0x1p11f;
__device__ __forceinline__ float terms_sum(float first, float others) { return __builtin_fmaf(others, 1.0f / kLowerTerms, first); }

// scales and bias of some channels or tokens: every type's loads in a branch of its own, so that they are in flight together
template <int kCount>
__device__ __forceinline__ void load_scales(const void *p, int f16, const int64_t (&at)[kCount], float (&s)[kCount])
{
    if (f16) {
#pragma unroll
        for (int c = 0; c < kCount; ++c) s[c] = __half2float(((const __half *)p)[at[c]]);
    } else {
#pragma unroll
        for (int c = 0; c < kCount; ++c) s[c] = ((const float *)p)[at[c]];
    }
}
template <int kCount>
__device__ __forceinline__ void channel_bias(const LinearArgs &A, const int64_t (&at)[kCount], float (&b)[kCount])
{
    if (!A.bias) {
#pragma unroll
        for (int c = 0; c < kCount; ++c) b[c] = 0.0f;
    } else if (A.dtype == BQ_F32) {
#pragma unroll
        for (int c = 0; c < kCount; ++c) b[c] = ((const float *)A.bias)[at[c]];
    } else if (A.dtype == BQ_F16) {
#pragma unroll
        for (int c = 0; c < kCount; ++c) b[c] = __half2float(((const __half *)A.bias)[at[c]]);
    } else {
#pragma unroll
        for (int c = 0; c < kCount; ++c) b[c] = to_float(((const bf16_t *)A.bias)[at[c]]);
    }
}

// kCount (a multiple of 4) consecutive results of one row at any address, `left` of them inside the row
template <int kCount>
__device__ __forceinline__ void store_results(const LinearArgs &A, int64_t at, const float (&v)[kCount], int left)
{
    if (left >= kCount) {
        if (A.dtype == BQ_F32) {
#pragma unroll
            for (int j = 0; j < kCount; j += 4) __builtin_memcpy((float *)A.y + at + j, v + j, 16);
            return;
        }
        uint32_t w[kCount / 2];
#pragma unroll
        for (int j = 0; j < kCount; j += 2)
            w[j / 2] = A.dtype == BQ_F16 ? f32x2_to_f16x2_bits(v[j], v[j + 1]) : f32x2_to_bf16x2_bits(v[j], v[j + 1]);
        uint16_t *p = (uint16_t *)A.y + at;
        if constexpr (kCount % 8 == 0) {
#pragma unroll
            for (int j = 0; j < kCount / 2; j += 4) __builtin_memcpy(p + 2 * j, w + j, 16);
        } else {
#pragma unroll
            for (int j = 0; j < kCount / 2; j += 2) __builtin_memcpy(p + 2 * j, w + j, 8);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kCount; ++j)
        if (j < left) store_row_value(A.y, at + j, A.dtype, v[j]);
}

}  // namespace bq
