// The product for any width, stride and alignment: a workgroup of four waves takes 64 tokens x 64 channels, its threads fetch the
// codes one by one and lay them out as bytes in LDS.  Bound by those loads: 8-bit codes 4096 -> 4096, rows 4097 bytes apart, 16 tokens 300 us, 2048
// tokens 1.6 ms (43 TOP/s).  The shapes of real layers go to the other kernels, and so do
// all gradients, whose rows are padded.
#include "bq_linear.h"

namespace bq {

namespace {

constexpr int kTile = 64, kStep = 64, kLd = kStep + 16;  // (rows 80 bytes apart: the 16-byte reads of 16 rows spread over the banks)

__device__ __forceinline__ uint8_t code_at(const uint8_t *row, int k, int bits)
{
    if (bits == 8) return row[k];
    if (bits == 4) return (uint8_t)((row[k >> 1] >> ((k & 1) * 4)) << 4);
    return (uint8_t)((row[k >> 2] >> ((k & 3) * 2)) << 6);
}

__global__ __launch_bounds__(256) void linear_any_kernel(LinearArgs A, int xbits, int wbits)
{
    __shared__ __align__(16) uint8_t s_x[kTile * kLd], s_w[kTile * kLd];
    const int n_tiles = (A.n + kTile - 1) / kTile;
    const RowTile rt = row_tile(A, blockIdx.x / n_tiles, kTile);
    if (rt.row0 >= rt.row_end) return;
    const int o0 = (int)(blockIdx.x % n_tiles) * kTile;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int to = (wave & 1) * 32, tt = (wave >> 1) * 32;  // this wave's 32 channels x 32 tokens
    const int r16 = lane & 15, kq = (lane >> 4) * 16;
    const int srow = tid >> 2, sk = (tid & 3) * 16;  // the 16 codes this thread fetches
    const int64_t token = rt.row0 + srow;
    const bool has_token = token < rt.row_end, has_channel = o0 + srow < A.n;
    const uint8_t *wrow = A.w + rt.expert * A.w_step + (int64_t)(o0 + srow) * A.ldw, *xrow = A.x + token * A.ldx;
    i32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < A.k; k0 += kStep) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int k = k0 + sk + j;
            s_x[srow * kLd + sk + j] = has_token && k < A.k ? code_at(xrow, k, xbits) : 0;
            s_w[srow * kLd + sk + j] = has_channel && k < A.k ? code_at(wrow, k, wbits) : 0;
        }
        __syncthreads();
        i32x4 w[2], x[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            w[i] = *(const i32x4 *)(s_w + (to + 16 * i + r16) * kLd + kq);
            x[i] = *(const i32x4 *)(s_x + (tt + 16 * i + r16) * kLd + kq);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t t = rt.row0 + tt + 16 * j + r16;
        if (t >= rt.row_end) continue;
        const float xs = load_scale(A.xs, t, A.xs_f16);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int o = o0 + to + 16 * i + (lane >> 4) * 4 + r;
                if (o >= A.n) continue;
                const int64_t at = (int64_t)rt.expert * A.n + o;
                float v = (float)acc[i][j][r] * A.factor * xs * load_scale(A.ws, at, A.ws_f16);
                if (A.bias) v += load_row_value(A.bias, at, A.dtype);
                store_row_value(A.y, t * A.ldy + o, A.dtype, v);
            }
    }
}

}  // namespace

hipError_t launch_linear_any(const LinearArgs &A, int xbits, int wbits, hipStream_t stream)
{
    const int64_t blocks = row_tiles_bound(A, kTile) * ((A.n + kTile - 1) / kTile);
    hipLaunchKernelGGL(linear_any_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, A, xbits, wbits);
    return hipGetLastError();
}

}  // namespace bq
