// What the gradient of a quantised product needs in front of the product itself: dy times the weights' scales as digits, and the
// weights' codes transposed, both with the summed index (the layer's outputs) contiguous and padded with zeros.
//
// Digits.  v = dy ws is written as  v = f (256 d1 + d0)  (16-bit rows) or  f (65536 d2 + 256 d1 + d0)  (float32 rows), digits in
// [-128, 127], f = max |v| / m with m = 32639 or 8355711, the largest number whose digits fit.  That rounds every term of the sum to
// half of f: 2^-16 or 2^-24 of the row's largest term, against the 2^-9 or 2^-12 of the term itself that a product in the row's type
// would leave.  Digits cost the matrix cores less than they look: two products of 8 bits take the time of one of 16 bits.  A row
// with an infinity or NaN gets f = NaN: its gradient is NaN throughout.
#include "bq_cascade.h"
#include "bq_linear.h"

namespace bq {

namespace {

struct DigitArgs {
    const void *dy, *ws;
    int8_t *planes;   // [kPlanes][rows][np]
    float *factor;    // [rows]
    const int32_t *offsets;
    int64_t rows, ld_dy;
    int n, np, experts, ws_f16;
};

__device__ __forceinline__ uint32_t block_max(uint32_t m)
{
    __shared__ uint32_t s_max[4];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)m, d, 64);
        m = m > o ? m : o;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) m = m > s_max[w] ? m : s_max[w];
    return m;
}

// The expert of a row, -1 if it has none; the whole wave asks for the same row.
__device__ __forceinline__ int expert_of(const int32_t *offsets, int experts, int64_t row)
{
    if (!offsets) return 0;
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < experts; base += 64) {
        const int e = base + lane;
        const bool in = e < experts && offsets[e] <= row && row < offsets[e + 1];
        const unsigned long long hit = __ballot(in);
        if (hit) return base + __ffsll(hit) - 1;
    }
    return -1;
}

template <typename T, int kPlanes>
__global__ __launch_bounds__(256) void linear_digits_kernel(DigitArgs A, int vec)
{
    constexpr float kMost = kPlanes == 3 ? 8355711.0f : 32639.0f;
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const int expert = expert_of(A.offsets, A.experts, row);
        if (expert < 0) continue;  // (the product does not look at it)
        const T *dy = (const T *)A.dy + row * A.ld_dy;
        const int64_t s0 = (int64_t)expert * A.n;
        auto eight = [&](int c, float (&v)[8]) {  // dy ws of 8 channels, 0 behind the last
            if (vec && c + 8 <= A.n) {
                unpack8(load8(dy + c), v, (const T *)nullptr);
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] *= load_scale(A.ws, s0 + c + r, A.ws_f16);
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = c + r < A.n ? to_float(dy[c + r]) * load_scale(A.ws, s0 + c + r, A.ws_f16) : 0.0f;
            }
        };
        uint32_t m = 0;
        for (int c = threadIdx.x * 8; c < A.n; c += 2048) {
            float v[8];
            eight(c, v);
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const uint32_t b = __float_as_uint(v[r]) & 0x7FFFFFFFu;
                m = m > b ? m : b;
            }
        }
        m = block_max(m);
        const bool finite = m < 0x7F800000u;
        const float amax = __uint_as_float(m);
        // rows of tiny entries are lifted first: m / amax has to be a float32 number
        const float lift = amax < 0x1p-60f ? 0x1p60f : 1.0f;
        const float top = amax * lift;
        const bool some = finite && top >= 0x1p-60f;  // (below 2^-120 the row counts as 0)
        const float inv = some ? kMost / top : 0.0f;
        if (threadIdx.x == 0) A.factor[row] = !finite ? __uint_as_float(0x7FC00000u) : some ? (top / kMost) / lift : 0.0f;
        for (int c = threadIdx.x * 8; c < A.np; c += 2048) {
            float v[8];
            eight(c, v);
            uint32_t d[kPlanes][2] = {};
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const float q = rintf(v[r] * lift * inv);
                const int u = some ? (int)fminf(fmaxf(q, -kMost), kMost) : 0;
                const int low = (u + 128) >> 8;  // u without its lowest digit, over 256
                const int sh = (r & 3) * 8;
                d[kPlanes - 1][r >> 2] |= ((uint32_t)(u - low * 256) & 255u) << sh;
                if (kPlanes == 3) {
                    const int high = (low + 128) >> 8;
                    d[kPlanes - 2][r >> 2] |= ((uint32_t)(low - high * 256) & 255u) << sh;
                    d[0][r >> 2] |= ((uint32_t)high & 255u) << sh;
                } else {
                    d[0][r >> 2] |= ((uint32_t)low & 255u) << sh;
                }
            }
#pragma unroll
            for (int p = 0; p < kPlanes; ++p)
                *(uint2 *)(A.planes + ((int64_t)p * A.rows + row) * A.np + c) = make_uint2(d[p][0], d[p][1]);
        }
    }
}

struct TransposeArgs {
    const uint8_t *w;
    int8_t *out;  // [experts][k][np]
    const int32_t *offsets;
    int64_t ldw, w_step;
    int n, k, np, bits, vec;
};

constexpr int kTr = 64;

// 64 outputs x 64 inputs per workgroup through LDS; codes of 4 and 2 bits come out as whole bytes.
__global__ __launch_bounds__(256) void linear_transpose_kernel(TransposeArgs A)
{
    __shared__ __align__(16) uint8_t s[kTr][kTr + 4];
    const int expert = blockIdx.z;
    if (A.offsets && A.offsets[expert + 1] <= A.offsets[expert]) return;  // no rows
    const int k0 = blockIdx.x * kTr, o0 = blockIdx.y * kTr;
    const int row = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;
    const uint8_t *w = A.w + expert * A.w_step + (int64_t)(o0 + row) * A.ldw;
    uint32_t c[4] = {};
    if (o0 + row < A.n) {
        if (A.vec && k0 + part + 16 <= A.k) {
            if (A.bits == 8) {
                const uint4 v = *(const uint4 *)(w + k0 + part);
                c[0] = v.x; c[1] = v.y; c[2] = v.z; c[3] = v.w;
            } else {
                const int per = 8 / A.bits;
                const uint8_t *p = w + (k0 + part) / per;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int f = (int)(int8_t)(uint8_t)(p[j / per] << (8 - A.bits - (j % per) * A.bits)) >> (8 - A.bits);
                    c[j >> 2] |= ((uint32_t)f & 255u) << ((j & 3) * 8);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int k = k0 + part + j;
                if (k >= A.k) continue;
                const int per = 8 / A.bits;
                const int f = (int)(int8_t)(uint8_t)(w[k / per] << (8 - A.bits - (k % per) * A.bits)) >> (8 - A.bits);
                c[j >> 2] |= ((uint32_t)f & 255u) << ((j & 3) * 8);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) *(uint32_t *)&s[row][part + 4 * j] = c[j];
    __syncthreads();
    const int k = k0 + row;  // now a row of the result
    if (k >= A.k) return;
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        r[j] = (uint32_t)s[part + 4 * j][row] | (uint32_t)s[part + 4 * j + 1][row] << 8 | (uint32_t)s[part + 4 * j + 2][row] << 16 |
               (uint32_t)s[part + 4 * j + 3][row] << 24;
    *(uint4 *)(A.out + ((int64_t)expert * A.k + k) * A.np + o0 + part) = make_uint4(r[0], r[1], r[2], r[3]);
}

int padded(int n) { return (n + 127) / 128 * 128; }

template <typename T, int kPlanes>
hipError_t launch_digits(const DigitArgs &D, hipStream_t stream)
{
    const int vec = (uintptr_t)D.dy % 16 == 0 && D.ld_dy * sizeof(T) % 16 == 0;
    hipLaunchKernelGGL((linear_digits_kernel<T, kPlanes>), dim3((unsigned)(D.rows < 65536 ? D.rows : 65536)), dim3(256), 0, stream, D, vec);
    return hipGetLastError();
}

}  // namespace

int linear_planes(int dtype) { return dtype == BQ_F32 ? 3 : 2; }

LinearBwdLayout linear_bwd_layout(int64_t rows, int n, int k, int experts, int dtype)
{
    LinearBwdLayout L;
    const size_t np = (size_t)padded(n);
    L.factor = 0;
    L.planes = align256((size_t)rows * sizeof(float));
    L.weights = L.planes + align256((size_t)linear_planes(dtype) * (size_t)rows * np);
    L.total = L.weights + align256((size_t)experts * (size_t)k * np);
    return L;
}

hipError_t launch_linear_bwd(const void *dy, int64_t ld_dy, const void *w, int wbits, int64_t ldw, const void *ws, int ws_f16,
                             const int32_t *offsets, void *dx, int64_t ld_dx, void *workspace, int64_t rows, int n, int k, int experts,
                             int dtype, hipStream_t stream)
{
    const LinearBwdLayout L = linear_bwd_layout(rows, n, k, experts, dtype);
    char *base = (char *)workspace;
    const int np = padded(n), planes = linear_planes(dtype);
    DigitArgs D{};
    D.dy = dy;
    D.ws = ws;
    D.planes = (int8_t *)(base + L.planes);
    D.factor = (float *)(base + L.factor);
    D.offsets = offsets;
    D.rows = rows;
    D.ld_dy = ld_dy;
    D.n = n;
    D.np = np;
    D.experts = experts;
    D.ws_f16 = ws_f16;
    hipError_t e = dtype == BQ_F32   ? launch_digits<float, 3>(D, stream)
                   : dtype == BQ_F16 ? launch_digits<__half, 2>(D, stream)
                                     : launch_digits<bf16_t, 2>(D, stream);
    if (e != hipSuccess) return e;
    TransposeArgs R{};
    R.w = (const uint8_t *)w;
    R.out = (int8_t *)(base + L.weights);
    R.offsets = offsets;
    R.ldw = ldw;
    R.w_step = (int64_t)n * ldw;
    R.n = n;
    R.k = k;
    R.np = np;
    R.bits = wbits;
    R.vec = (uintptr_t)w % 16 == 0 && ldw % 16 == 0;
    hipLaunchKernelGGL(linear_transpose_kernel, dim3((unsigned)((k + kTr - 1) / kTr), (unsigned)(np / kTr), (unsigned)experts), dim3(256), 0,
                       stream, R);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    LinearArgs A{};
    A.x = (const uint8_t *)(base + L.planes);
    A.w = (const uint8_t *)(base + L.weights);
    A.xs = base + L.factor;
    A.y = dx;
    A.offsets = offsets;
    A.rows = rows;
    A.ldx = A.ldw = np;
    A.ldy = ld_dx;
    A.w_step = (int64_t)k * np;
    A.plane_step = rows * np;
    A.k = np;
    A.n = k;
    A.experts = experts;
    A.dtype = dtype;
    A.factor = 1.0f;
    return launch_linear(A, 8, 8, planes, stream);
}

}  // namespace bq
