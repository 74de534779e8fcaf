// The product for few rows (decoding): the weights' bytes are the work.  A workgroup of 8 waves takes 16 channels and all tokens of
// its block; the waves share the sum's index, step by step, so that the workgroup reads its channels' codes front to back, every
// code once and straight into the registers the matrix instruction reads (16 bytes of one channel per lane).  The 8 partial sums are
// joined through LDS, in integers: the order does not matter.
#pragma once

#include "bq_linear_codes.h"

namespace bq {

constexpr int kRowsWaves = 8;

// kBlocks: 16-token blocks per pass
template <int kXBits, int kWBits, int kPlanes, int kBlocks>
__global__ __launch_bounds__(64 * kRowsWaves) void linear_rows_kernel(LinearArgs A)
{
    constexpr int kFrags = kBlocks * kPlanes;
    constexpr int kCodes = 128 / kWBits;       // codes of a lane per step: one 16-byte load of weights
    constexpr int kSub = kCodes / 16;          // matrix instructions per step and 16 tokens
    constexpr int kXWords = kCodes * kXBits / 32;
    constexpr int kAhead = kFrags * kXWords <= 4 ? 8 : kFrags * kXWords <= 8 ? 4 : 2;  // steps whose loads are in flight together
    constexpr bool kNatural = kXBits != kWBits;
    __shared__ i32x4 s_part[kRowsWaves][kFrags][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16;
    const int expert = A.offsets ? blockIdx.y : 0;
    int64_t row_a, row_b;
    expert_rows(A, expert, &row_a, &row_b);
    const int channel = o0 + r16 < A.n ? o0 + r16 : A.n - 1;
    const uint8_t *w = A.w + expert * A.w_step + (int64_t)channel * A.ldw;
    const int steps = (A.k + 4 * kCodes - 1) / (4 * kCodes);
    const int64_t pass = 16 * kBlocks;
    for (int64_t row0 = row_a + (A.offsets ? 0 : blockIdx.y * pass); row0 < row_b; row0 += A.offsets ? pass : gridDim.y * pass) {
        const uint8_t *x[kFrags];
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const int64_t t = row0 + 16 * (f / kPlanes) + r16;
            x[f] = A.x + (f % kPlanes) * A.plane_step + (t < row_b ? t : row_b - 1) * A.ldx;
        }
        i32x4 acc[kFrags] = {};
        for (int s0 = wave; s0 < steps; s0 += kRowsWaves * kAhead) {
            uint32_t wv[kAhead][4], xv[kAhead][kFrags][kXWords];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int k = (s0 + u * kRowsWaves) * 4 * kCodes + g * kCodes;
                const bool in = k < A.k;  // (a lane's codes are all inside or all outside)
                const uint4 q = *(const uint4 *)(w + (in ? (int64_t)k * kWBits / 8 : 0));
                wv[u][0] = in ? q.x : 0; wv[u][1] = in ? q.y : 0; wv[u][2] = in ? q.z : 0; wv[u][3] = in ? q.w : 0;
                const int64_t xo = in ? (int64_t)k * kXBits / 8 : 0;
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
                    const i32x4 a = step_codes<kWBits, kNatural>(wv[u], s);
#pragma unroll
                    for (int f = 0; f < kFrags; ++f)
                        acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, step_codes<kXBits, kNatural>(xv[u][f], s), acc[f], 0, 0, 0);
                }
        }
        __syncthreads();  // (the last pass's sums have been read)
#pragma unroll
        for (int f = 0; f < kFrags; ++f) s_part[wave][f][lane] = acc[f];
        __syncthreads();
        if (wave >= kBlocks) continue;
        i32x4 sum[kPlanes];
#pragma unroll
        for (int p = 0; p < kPlanes; ++p) {
            sum[p] = s_part[0][wave * kPlanes + p][lane];
#pragma unroll
            for (int v = 1; v < kRowsWaves; ++v) sum[p] += s_part[v][wave * kPlanes + p][lane];
        }
        const int64_t t = row0 + 16 * wave + r16;
        const int o = o0 + 4 * g;
        if (t >= row_b || o >= A.n) continue;
        const float xs = load_scale(A.xs, t, A.xs_f16) * A.factor;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t at = (int64_t)expert * A.n + (o + r < A.n ? o + r : A.n - 1);
            int part[kPlanes];
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) part[p] = sum[p][r];
            v[r] = joined<kPlanes>(part) * xs;
            if (A.ws) v[r] *= load_scale(A.ws, at, A.ws_f16);
            if (A.bias) v[r] += load_row_value(A.bias, at, A.dtype);
        }
        store_results<4>(A, t * A.ldy + o, v, A.n - o, A.y_quads);
    }
}

template <int kXBits, int kWBits, int kPlanes>
hipError_t launch_rows(const LinearArgs &A, int blocks, hipStream_t stream)
{
    const unsigned columns = (unsigned)((A.n + 15) / 16);
    const unsigned passes = A.offsets ? (unsigned)A.experts : (unsigned)((A.rows + 16 * blocks - 1) / (16 * blocks));
    const dim3 grid(columns, passes), threads(64 * kRowsWaves);
    if (blocks == 1)
        hipLaunchKernelGGL((linear_rows_kernel<kXBits, kWBits, kPlanes, 1>), grid, threads, 0, stream, A);
    else if (blocks == 2 || kPlanes > 1)
        hipLaunchKernelGGL((linear_rows_kernel<kXBits, kWBits, kPlanes, 2>), grid, threads, 0, stream, A);
    else if constexpr (kPlanes == 1)
        hipLaunchKernelGGL((linear_rows_kernel<kXBits, kWBits, kPlanes, 4>), grid, threads, 0, stream, A);
    return hipGetLastError();
}

}  // namespace bq
