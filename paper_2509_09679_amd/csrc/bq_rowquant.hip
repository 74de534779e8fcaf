// INT8 codes and one scale per row:  s = max |x| / 127,  q = clip(rint(x / s)).  One read of the rows, one write of the codes:
// bound by HBM.  A row's entries stay in registers between the maximum and the codes; rows share a wave, have one, or a workgroup.  bf16:
// 32768 x 4096 68 us (5.9 TB/s), 524288 x 128 39 us (5.2 TB/s), 10000 x 5063 43 us (3.5 TB/s); float32: 1777 x 5120 8.5 us (5.3 TB/s).
#include <type_traits>

#include "bq_linear.h"
#include "bq_piece.h"

namespace bq {

namespace {

template <int kN>
using N = std::integral_constant<int, kN>;

struct RowQuantArgs {
    const void *x;
    int8_t *codes;
    void *scales;
    int64_t rows, ld_x, ld_codes;
    int cols, scale_f16;
};

// The scale of a row from the bit pattern of its largest magnitude (patterns of non-negative floats are ordered like their
// values, infinity and NaN above all): a row that holds one of those gets the scale NaN and codes 0, so that a product with it
// is NaN instead of a plausible number.  A scale below 2^-126, whose reciprocal float32 cannot hold, counts as 0.
__device__ __forceinline__ float row_scale(uint32_t amax_bits, int scale_f16, float *inv)
{
    if (amax_bits >= 0x7F800000u) {
        *inv = 0.0f;
        return __uint_as_float(0x7FC00000u);
    }
    float s = __uint_as_float(amax_bits) / 127.0f;
    if (scale_f16) s = __half2float(__float2half_rn(fminf(s, 65504.0f)));
    if (s < 1.17549435e-38f) s = 0.0f;
    *inv = s == 0.0f ? 0.0f : 1.0f / s;
    return s;
}

__device__ __forceinline__ int code8(float v, float inv)
{
    const float q = rintf(v * inv);  // (inv is 0 on rows with infinities: 0 * inf is NaN, which the clip takes to -128)
    return inv == 0.0f ? 0 : (int)fminf(fmaxf(q, -128.0f), 127.0f);
}

template <int kLanes>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m)
{
#pragma unroll
    for (int d = 1; d < (kLanes < 64 ? kLanes : 64); d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)m, d, 64);
        m = m > o ? m : o;
    }
    return m;
}

// kLanes threads per row (16 .. 64: several rows per workgroup), kPasses pieces of 8 elements per thread.  kWhole: a
// row's pieces are whole (with a branch for the last one between the loads, 1777 rows of 5120 take 9.5 us instead of 8.6 us).
template <typename T, int kLanes, int kPasses, bool kWhole>
__global__ __launch_bounds__(kLanes < 256 ? 256 : kLanes) void row_quant_kernel(RowQuantArgs A)
{
    constexpr int kThreads = kLanes < 256 ? 256 : kLanes, kRows = kThreads / kLanes;
    __shared__ uint32_t s_max[kThreads / 64];
    const int lane = threadIdx.x % kLanes;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + threadIdx.x / kLanes;
    const bool live = row < A.rows;
    const T *x = (const T *)A.x + (live ? row : 0) * A.ld_x;
    float v[kPasses][8];
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int c = (p * kLanes + lane) * 8;
#pragma unroll
        for (int r = 0; r < 8; ++r) v[p][r] = 0.0f;
        if (live && c < A.cols) unpack8(kWhole ? load_whole_piece(x + c) : load_piece(x + c, A.cols - c), v[p], (const T *)nullptr);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint32_t b = __float_as_uint(v[p][r]) & 0x7FFFFFFFu;
            m = m > b ? m : b;
        }
    }
    m = lanes_max<kLanes>(m);
    if (kLanes > 64) {
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) m = m > s_max[w] ? m : s_max[w];
    }
    if (!live) return;
    float inv;
    const float s = row_scale(m, A.scale_f16, &inv);
    if (lane == 0) {
        if (A.scale_f16)
            ((__half *)A.scales)[row] = __float2half_rn(s);
        else
            ((float *)A.scales)[row] = s;
    }
    int8_t *out = A.codes + row * A.ld_codes;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int c = (p * kLanes + lane) * 8;
        if (c >= A.cols) continue;
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            w[h] = ((uint32_t)code8(v[p][4 * h], inv) & 255u) | ((uint32_t)code8(v[p][4 * h + 1], inv) & 255u) << 8 |
                   ((uint32_t)code8(v[p][4 * h + 2], inv) & 255u) << 16 | (uint32_t)code8(v[p][4 * h + 3], inv) << 24;
        store_piece(out + c, make_uint2(w[0], w[1]), kWhole ? 8 : A.cols - c);
    }
}

// Wider rows, one workgroup each; the second look at the row comes from the caches.
template <typename T>
__global__ __launch_bounds__(256) void row_quant_wide_kernel(RowQuantArgs A)
{
    __shared__ uint32_t s_max[4];
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const T *x = (const T *)A.x + row * A.ld_x;
        uint32_t m = 0;
        for (int c = threadIdx.x; c < A.cols; c += 256) {
            const uint32_t b = __float_as_uint(to_float(x[c])) & 0x7FFFFFFFu;
            m = m > b ? m : b;
        }
        m = lanes_max<64>(m);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) m = m > s_max[w] ? m : s_max[w];
        float inv;
        const float s = row_scale(m, A.scale_f16, &inv);
        if (threadIdx.x == 0) {
            if (A.scale_f16)
                ((__half *)A.scales)[row] = __float2half_rn(s);
            else
                ((float *)A.scales)[row] = s;
        }
        int8_t *out = A.codes + row * A.ld_codes;
        for (int c = threadIdx.x; c < A.cols; c += 256) out[c] = (int8_t)code8(to_float(x[c]), inv);
    }
}

template <typename T>
hipError_t launch_typed(const RowQuantArgs &A, hipStream_t stream)
{
    if (A.cols > 32768) {
        hipLaunchKernelGGL(row_quant_wide_kernel<T>, dim3((unsigned)(A.rows < 65536 ? A.rows : 65536)), dim3(256), 0, stream, A);
        return hipGetLastError();
    }
    auto launch = [&](auto LANES, auto PASSES) {
        constexpr int lanes = decltype(LANES)::value, passes = decltype(PASSES)::value, threads = lanes < 256 ? 256 : lanes;
        // (threads along a dimension of a launch are counted in 32 bits)
        const int64_t groups = (A.rows + threads / lanes - 1) / (threads / lanes);
        const dim3 grid((unsigned)(groups < 1 << 20 ? groups : 1 << 20), (unsigned)((groups + (1 << 20) - 1) >> 20));
        if (A.cols % 8 == 0)
            hipLaunchKernelGGL((row_quant_kernel<T, lanes, passes, true>), grid, dim3(threads), 0, stream, A);
        else
            hipLaunchKernelGGL((row_quant_kernel<T, lanes, passes, false>), grid, dim3(threads), 0, stream, A);
        return hipGetLastError();
    };
    const int eights = (A.cols + 7) / 8;
    if (eights <= 16) return launch(N<16>{}, N<1>{});
    if (eights <= 32) return launch(N<32>{}, N<1>{});
    if (eights <= 64) return launch(N<64>{}, N<1>{});
    if (eights <= 128) return launch(N<64>{}, N<2>{});
    if (eights <= 256) return launch(N<256>{}, N<1>{});
    if (eights <= 512) return launch(N<256>{}, N<2>{});
    if (eights <= 1024) return launch(N<256>{}, N<4>{});
    if (eights <= 2048) return launch(N<512>{}, N<4>{});
    return launch(N<1024>{}, N<4>{});
}

}  // namespace

hipError_t launch_row_quant(const void *x, int64_t rows, int cols, int64_t ld_x, int dtype, int8_t *codes, int64_t ld_codes, void *scales,
                            int scale_f16, hipStream_t stream)
{
    RowQuantArgs A{x, codes, scales, rows, ld_x, ld_codes, cols, scale_f16};
    if (dtype == BQ_F32) return launch_typed<float>(A, stream);
    if (dtype == BQ_F16) return launch_typed<__half>(A, stream);
    return launch_typed<bf16_t>(A, stream);
}

}  // namespace bq
