// The product for few rows.  A workgroup of 8 waves takes kBlocks x kCols pieces of 16 tokens x 16 channels; the waves share the sum's
// index, step by step, so that the workgroup reads its channels' codes front to back, every code once and straight into the registers
// that the matrix instruction reads (16 bytes of one channel per lane).  The 8 partial sums are joined through LDS, in integers: the
// order does not matter.  Decoding (a few tokens, kCols = 1) is bound by the weights' bytes; with more tokens the pieces grow, since a
// code of x is read once per kCols pieces and one of w once per kBlocks.
#pragma once

#include "bq_linear_codes.h"

namespace bq {

constexpr int kRowsWaves = 8;

template <int kXBits, int kWBits, int kPlanes, int kBlocks, int kCols>
__global__ __launch_bounds__(64 * kRowsWaves) void linear_rows_kernel(LinearArgs A)
{
    constexpr int kFrags = kBlocks * kPlanes;
    constexpr int kCodes = 128 / kWBits;       // codes of a lane per step: one 16-byte load of weights
    constexpr int kSub = kCodes / 16;          // matrix instructions per step and piece
    constexpr int kXWords = kCodes * kXBits / 32;
    constexpr int kWords = kFrags * kXWords + kCols * 4;  // registers that a step's loads fill
    // steps whose loads are in flight together (swept: 8-bit weights gain from more, 6.1 us against 7.2 with two steps for one token
    // 4096 -> 4096; packed ones lose, 9.7 against 8.8 us for one token 4096 -> 11008 with four)
    constexpr int kAhead = kWBits == 8 && kWords <= 8 ? 8 : kWBits == 8 && kWords <= 12 ? 4 : kWords <= 40 ? 2 : 1;
    constexpr int kPairs = kBlocks * kCols, kChunk = kPairs < 8 / kPlanes ? kPairs : 8 / kPlanes;  // pieces joined at a time: 64 KB
    constexpr bool kNatural = kXBits != kWBits;
    __shared__ i32x4 s_part[kRowsWaves][kChunk * kPlanes][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16 * kCols;
    const int expert = A.offsets ? blockIdx.z : 0;
    int64_t row_a, row_b;
    expert_rows(A, expert, &row_a, &row_b);
    const uint8_t *w[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        const int channel = o0 + 16 * c + r16;
        w[c] = A.w + expert * A.w_step + (int64_t)(channel < A.n ? channel : A.n - 1) * A.ldw;
    }
    const int steps = (A.k + 4 * kCodes - 1) / (4 * kCodes);
    const int64_t pass = 16 * kBlocks;
    for (int64_t row0 = row_a + blockIdx.y * pass; row0 < row_b; row0 += gridDim.y * pass) {
        const uint8_t *x[kFrags];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const int64_t t = row0 + 16 * (f / kPlanes) + r16;
            x[f] = A.x + (f % kPlanes) * A.plane_step + (t < row_b ? t : row_b - 1) * A.ldx;
        }
        i32x4 acc[kCols][kFrags] = {};
        for (int s0 = wave; s0 < steps; s0 += kRowsWaves * kAhead) {
            uint32_t wv[kAhead][kCols][4], xv[kAhead][kFrags][kXWords];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int k = (s0 + u * kRowsWaves) * 4 * kCodes + g * kCodes;
                const bool in = k < A.k;  // (a lane's codes are all inside or all outside)
                const int wo = in ? (int)((int64_t)k * kWBits / 8) : 0, xo = in ? (int)((int64_t)k * kXBits / 8) : 0;
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const uint4 q = *(const uint4 *)(w[c] + wo);
                    wv[u][c][0] = in ? q.x : 0; wv[u][c][1] = in ? q.y : 0; wv[u][c][2] = in ? q.z : 0; wv[u][c][3] = in ? q.w : 0;
                }
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    if constexpr (kXWords == 2) {
                        const uint2 p = *(const uint2 *)(x[f] + xo);
                        xv[u][f][0] = p.x; xv[u][f][1] = p.y;
                    } else {
#pragma unroll
                        for (int j = 0; j < kXWords; j += 4) {
                            const uint4 p = *(const uint4 *)(x[f] + xo + 4 * j);
                            xv[u][f][j] = p.x; xv[u][f][j + 1] = p.y; xv[u][f][j + 2] = p.z; xv[u][f][j + 3] = p.w;
                        }
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int s = 0; s < kSub; ++s) {
                    i32x4 a[kCols];
#pragma unroll
                    for (int c = 0; c < kCols; ++c) a[c] = step_codes<kWBits, kNatural>(wv[u][c], s);
#pragma unroll
                    for (int f = 0; f < kFrags; ++f) {
                        const i32x4 b = step_codes<kXBits, kNatural>(xv[u][f], s);
#pragma unroll
                        for (int c = 0; c < kCols; ++c) acc[c][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[c], b, acc[c][f], 0, 0, 0);
                    }
                }
        }
#pragma unroll
        for (int first = 0; first < kPairs; first += kChunk) {
            __syncthreads();  // (the sums before have been read)
#pragma unroll
            for (int i = 0; i < kChunk; ++i)
#pragma unroll
                for (int p = 0; p < kPlanes; ++p)
                    if (first + i < kPairs) s_part[wave][i * kPlanes + p][lane] = acc[(first + i) / kBlocks][(first + i) % kBlocks * kPlanes + p];
            __syncthreads();
            const int pair = first + wave, block = pair % kBlocks, col = pair / kBlocks;
            if (wave >= kChunk || pair >= kPairs) continue;
            i32x4 sum[kPlanes];
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) {
                sum[p] = s_part[0][wave * kPlanes + p][lane];
#pragma unroll
                for (int v = 1; v < kRowsWaves; ++v) sum[p] += s_part[v][wave * kPlanes + p][lane];
            }
            const int64_t t = row0 + 16 * block + r16;
            const int o = o0 + 16 * col + 4 * g;
            if (t >= row_b || o >= A.n) continue;
            const float xs = load_scale(A.xs, t, A.xs_f16) * A.factor;
            int64_t at[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) at[r] = (int64_t)expert * A.n + (o + r < A.n ? o + r : A.n - 1);
            float ws[4], bias[4], v[4];
            channel_scales(A, at, ws);
            channel_bias(A, at, bias);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                int part[kPlanes];
#pragma unroll
                for (int p = 0; p < kPlanes; ++p) part[p] = sum[p][r];
                v[r] = joined<kPlanes>(part) * xs;
                if (A.ws) v[r] *= ws[r];
                if (A.bias) v[r] += bias[r];
            }
            store_results<4>(A, t * A.ldy + o, v, A.n - o, A.y_quads);
        }
    }
}

template <int kXBits, int kWBits, int kPlanes, int kBlocks, int kCols>
hipError_t launch_rows(const LinearArgs &A, hipStream_t stream)
{
    // by expert: as many workgroups along the rows as an expert needs that has twice its share; they go on where it has more
    const int64_t rows = A.offsets ? (2 * A.rows + A.experts - 1) / A.experts : A.rows;
    const int64_t passes = (rows + 16 * kBlocks - 1) / (16 * kBlocks);
    const dim3 grid((unsigned)((A.n + 16 * kCols - 1) / (16 * kCols)), (unsigned)(passes < 1024 ? passes : 1024), (unsigned)A.experts);
    hipLaunchKernelGGL((linear_rows_kernel<kXBits, kWBits, kPlanes, kBlocks, kCols>), grid, dim3(64 * kRowsWaves), 0, stream, A);
    return hipGetLastError();
}

// blocks x cols: 1x1, 1x2 (packed weights), 2x1, 2x2, 4x2, 4x4; of a gradient's planes 1x1, 2x1, 2x2 and 2x4 (two) or 1x4 (three)
template <int kXBits, int kWBits, int kPlanes>
hipError_t launch_rows_of(const LinearArgs &A, int blocks, int cols, hipStream_t stream)
{
    if constexpr (kPlanes == 1) {
        if (blocks == 4) return cols == 2 ? launch_rows<kXBits, kWBits, 1, 4, 2>(A, stream) : launch_rows<kXBits, kWBits, 1, 4, 4>(A, stream);
        if constexpr (kWBits < 8) {
            if (blocks == 1 && cols == 2) return launch_rows<kXBits, kWBits, 1, 1, 2>(A, stream);
        }
    }
    if constexpr (kPlanes == 2) {
        if (cols == 4) return launch_rows<kXBits, kWBits, 2, 2, 4>(A, stream);
    }
    if constexpr (kPlanes == 3) {
        if (cols == 4) return launch_rows<kXBits, kWBits, 3, 1, 4>(A, stream);
    } else {
        if (blocks == 2 && cols == 2) return launch_rows<kXBits, kWBits, kPlanes, 2, 2>(A, stream);
    }
    return blocks == 1 ? launch_rows<kXBits, kWBits, kPlanes, 1, 1>(A, stream) : launch_rows<kXBits, kWBits, kPlanes, 2, 1>(A, stream);
}

}  // namespace bq
