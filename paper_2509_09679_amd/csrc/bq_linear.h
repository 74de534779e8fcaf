// Products of quantised rows with quantised weights: what the translation units share.
//
//     y[t, o] = xs[t] ws[o] sum_k x[t, k] w[o, k] + bias[o]
//
// x and w are codes of 8, 4 or 2 bits, summed in int32 on the matrix cores (v_mfma_i32_16x16x64_i8): exact, in whatever order,
// as |x w| <= 2^14 and k < 2^17.  Packed codes are not sign-extended: a field is moved to the top of a byte, which makes it 16
// (4 bits) or 64 (2 bits) times its value, and the epilogue's factor takes that out again (exact, a power of two).
//
// The gradient of the rows, dx[t, k] = sum_o dy[t, o] ws[o] w[o, k], is a product of the same form: dy ws is written as a sum of two or
// three binary16 numbers, `terms` planes, and multiplied with the codes as binary16 numbers (exact) on v_mfma_f32_16x16x32_f16.
//
// The matrix instruction's first operand is the weights: a lane then holds consecutive channels of one token.
#pragma once

#include "bq_device.h"
#include "bq_linear_choice.h"

namespace bq {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

struct LinearArgs {
    const uint8_t *x, *w;
    const void *xs, *ws, *bias;  // xs: of a gradient the rows' exponents (int32), and no ws; bias may be NULL (0)
    void *y;
    const int32_t *offsets;  // [experts + 1], NULL: one expert that has all rows
    int64_t rows, ldx, ldw, ldy;  // ldx, ldw in bytes, ldy in elements
    int64_t w_step, plane_step;   // bytes from one expert's weights to the next one's, from one plane of x to the next
    int k, n, experts;
    int xs_f16, ws_f16, dtype;
    float factor;  // of the fields' positions
    int w_rows;    // of weights that lie across (bq_linear_tile.h): the summed index may be padded beyond it
};

inline LinearSize size_of(const LinearArgs &A) { return LinearSize{A.rows, A.k, A.n, A.experts, A.offsets != nullptr, A.w_rows}; }

// Rows of one expert that a workgroup takes: [row0, row_end), at most the tile's.
struct RowTile {
    int expert;
    int64_t row0, row_end;
};

// offsets come from the device: whatever they hold, a range stays within [0, rows]
__device__ __forceinline__ void expert_rows(const LinearArgs &A, int e, int64_t *a, int64_t *b)
{
    if (!A.offsets) {
        *a = 0;
        *b = A.rows;
        return;
    }
    const int64_t lo = A.offsets[e], hi = A.offsets[e + 1];
    *a = lo < 0 ? 0 : lo > A.rows ? A.rows : lo;
    *b = hi < *a ? *a : hi > A.rows ? A.rows : hi;
}

// a value that all lanes of the wave hold, in scalar registers
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}

// The m-th tile of `tile` rows, counted over all experts (every expert's last one may be short); row0 == row_end behind the last.
// The lanes of a wave look at 64 experts at a time.
__device__ __forceinline__ RowTile row_tile(const LinearArgs &A, int64_t m, int tile)
{
    RowTile r;
    if (!A.offsets) {
        r.expert = 0;
        r.row0 = m * tile < A.rows ? m * tile : A.rows;
        r.row_end = r.row0 + tile < A.rows ? r.row0 + tile : A.rows;
        return r;
    }
    r.expert = 0;
    r.row0 = r.row_end = 0;
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < A.experts; base += 64) {
        int64_t a = 0, b = 0;
        if (base + lane < A.experts) expert_rows(A, base + lane, &a, &b);
        const int mine = (int)((b - a + tile - 1) / tile);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (m < all) {
            const int at = __ffsll((unsigned long long)__ballot(m < upto)) - 1;  // the first lane whose tiles reach beyond m
            const int64_t before = __shfl(upto - mine, at, 64);
            const int64_t ea = ((int64_t)__shfl((int)(a >> 32), at, 64) << 32) | (uint32_t)__shfl((int)a, at, 64);
            const int64_t eb = ((int64_t)__shfl((int)(b >> 32), at, 64) << 32) | (uint32_t)__shfl((int)b, at, 64);
            r.expert = __builtin_amdgcn_readfirstlane(base + at);
            r.row0 = uniform(ea + (m - before) * tile);
            r.row_end = uniform(ea + (m - before + 1) * tile < eb ? ea + (m - before + 1) * tile : eb);
            return r;
        }
        m -= all;
    }
    return r;
}

// how many there are
__device__ __forceinline__ int64_t row_tiles(const LinearArgs &A, int tile)
{
    if (!A.offsets) return (A.rows + tile - 1) / tile;
    const int lane = threadIdx.x & 63;
    int64_t all = 0;
    for (int base = 0; base < A.experts; base += 64) {
        int64_t a = 0, b = 0;
        if (base + lane < A.experts) expert_rows(A, base + lane, &a, &b);
        int mine = (int)((b - a + tile - 1) / tile);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d, 64);
        all += __builtin_amdgcn_readfirstlane(mine);
    }
    return all;
}

// an upper bound that the host can state
__host__ __device__ inline int64_t row_tiles_bound(const LinearArgs &A, int tile)
{
    if (!A.offsets) return (A.rows + tile - 1) / tile;
    return A.rows / tile + (A.experts < A.rows ? A.experts : A.rows);
}

__device__ __forceinline__ float load_scale(const void *p, int64_t at, int f16)
{
    return f16 ? __half2float(((const __half *)p)[at]) : ((const float *)p)[at];
}

__device__ __forceinline__ float load_row_value(const void *p, int64_t at, int dtype)
{
    if (dtype == BQ_F32) return ((const float *)p)[at];
    if (dtype == BQ_F16) return __half2float(((const __half *)p)[at]);
    return to_float(((const bf16_t *)p)[at]);
}

__device__ __forceinline__ void store_row_value(void *p, int64_t at, int dtype, float v)
{
    if (dtype == BQ_F32)
        ((float *)p)[at] = v;
    else if (dtype == BQ_F16)
        ((__half *)p)[at] = __float2half_rn(v);
    else
        ((bf16_t *)p)[at] = from_float<bf16_t>(v);
}

// ---- launchers --------------------------------------------------------------------------------------------
hipError_t launch_linear_any(const LinearArgs &A, int xbits, int wbits, hipStream_t stream);  // bq_linear_any.hip
// few rows: bq_linear_rows.h; blocks x cols: 16-token blocks and 16-channel columns of a workgroup
hipError_t launch_linear_rows8(const LinearArgs &A, int wbits, int blocks, int cols, hipStream_t stream);
hipError_t launch_linear_rows4(const LinearArgs &A, int wbits, int blocks, int cols, hipStream_t stream);
hipError_t launch_linear_rows_terms(const LinearArgs &A, int terms, int blocks, int cols, hipStream_t stream);
// many: bq_linear_tile.h
hipError_t launch_linear_tile8(const LinearArgs &A, int wbits, LinearTile tile, hipStream_t stream);
hipError_t launch_linear_tile4(const LinearArgs &A, int wbits, LinearTile tile, hipStream_t stream);
hipError_t launch_linear_tile_terms(const LinearArgs &A, int terms, LinearTile tile, hipStream_t stream);
hipError_t launch_linear_tile_across(const LinearArgs &A, int wbits, int terms, LinearTile tile, hipStream_t stream);
// these pick the kernel (bq_linear.hip); a gradient has two or three terms
hipError_t launch_linear(const LinearArgs &A, int xbits, int wbits, hipStream_t stream);
hipError_t launch_linear_terms(const LinearArgs &A, int terms, hipStream_t stream);
// the gradient's product with the weights as the layer has them, [summed index][channel]; is it quicker than transposing them first?
bool linear_across_is_quicker(const LinearArgs &across, int wbits, int terms);
hipError_t launch_linear_across(const LinearArgs &A, int wbits, int terms, hipStream_t stream);

}  // namespace bq
