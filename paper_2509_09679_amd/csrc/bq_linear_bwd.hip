// What the gradient of a quantised product needs in front of the product itself: dy times the weights' scales as digits, and, where the
// product does not read them as they lie, the weights' codes transposed, both with the summed index (the layer's outputs) contiguous and
// padded with zeros.
//
// Digits.  v = dy ws is written as  v = f (256 d1 + d0)  (16-bit rows) or  f (65536 d2 + 256 d1 + d0)  (float32 rows), digits in
// [-128, 127], f = max |v| / m with m = 32639 or 8355711, the largest number whose digits fit.  That rounds every term of the sum to
// half of f: 2^-16 or 2^-24 of the row's largest term, against the 2^-9 or 2^-12 of the term itself that a product in the row's type
// would leave.  Digits cost the matrix cores less than they look: two products of 8 bits take the time of one of 16 bits.  A row
// with an infinity or NaN gets f = NaN: its gradient is NaN throughout.
#include <type_traits>

#include "bq_linear_codes.h"
#include "bq_piece.h"

namespace bq {

namespace {

struct DigitArgs {
    const void *dy, *ws;
    int8_t *planes;   // [kPlanes][rows][np]
    float *factor;    // [rows]
    const int32_t *offsets;
    int64_t rows, ld_dy;
    int n, np, experts, ws_f16;
    int odd_last;  // eight digits lie as 0, 2, 4, 6, 1, 3, 5, 7: how packed codes come out of a word with the fewest steps
};

// over a wave, or a workgroup of four
template <int kThreads>
__device__ __forceinline__ uint32_t max_over(uint32_t m)
{
    static_assert(kThreads == 64 || kThreads == 256, "a wave or a workgroup");
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)m, d, 64);
        m = m > o ? m : o;
    }
    if (kThreads == 64) return m;
    __shared__ uint32_t s_max[4];
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

// the factor of a row and what its entries are multiplied with, from the bit pattern of its largest magnitude
struct RowFactor {
    float lift, inv, factor;
};

template <int kPlanes>
__device__ __forceinline__ RowFactor row_factor(uint32_t amax_bits)
{
    constexpr float kMost = kPlanes == 3 ? 8355711.0f : 32639.0f;
    const bool finite = amax_bits < 0x7F800000u;
    const float amax = __uint_as_float(amax_bits);
    // rows of tiny entries are lifted first: m / amax and amax / m have to be float32 numbers with all their digits; the factor's sign says so
    RowFactor f;
    f.lift = amax < 0x1p-60f ? 0x1p60f : 1.0f;
    const float top = amax * f.lift;
    const bool some = finite && top >= 0x1p-60f;  // (below 2^-120 the row counts as 0)
    f.inv = some ? kMost / top : 0.0f;
    f.factor = !finite ? __uint_as_float(0x7FC00000u) : some ? (f.lift != 1.0f ? -top : top) / kMost : 0.0f;
    return f;
}

// The digits of 8 entries, packed by plane.  With u = rint(v inv) + 128 (+ 128 * 256), the digits are u's bytes, all but the highest less
// 128; for two digits one addition to 1.5 * 2^23 both rounds and leaves u in the low bytes (|v inv| stays below m + 1/2).  The digits of
// rows without a finite largest entry do not matter, those of a row that counts as 0 are 0.
template <int kPlanes>
__device__ __forceinline__ void digits8(float (&v)[8], const RowFactor &f, int odd_last, uint2 (&d)[kPlanes])
{
    constexpr float kMost = 8355711.0f;
    uint32_t u[8], w[kPlanes][2];
    if (f.lift != 1.0f) {
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] *= f.lift;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
        u[r] = kPlanes == 2 ? __float_as_uint(__builtin_fmaf(v[r], f.inv, 0x1.8p23f + 128.0f))
                            : (uint32_t)((int)__builtin_amdgcn_fmed3f(rintf(v[r] * f.inv), -kMost, kMost) + 0x8080);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t *q = u + 4 * h;
        const uint32_t a = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u), b = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);
        const uint32_t second = __builtin_amdgcn_perm(b, a, 0x07060302u);
        w[kPlanes - 1][h] = __builtin_amdgcn_perm(b, a, 0x05040100u) ^ 0x80808080u;
        w[kPlanes - 2][h] = kPlanes == 2 ? second : second ^ 0x80808080u;
        if (kPlanes == 3)
            w[0][h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0C0C0602u), __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0602u),
                                            0x05040100u);
    }
#pragma unroll
    for (int p = 0; p < kPlanes; ++p)
        d[p] = odd_last ? make_uint2(__builtin_amdgcn_perm(w[p][1], w[p][0], 0x06040200u), __builtin_amdgcn_perm(w[p][1], w[p][0], 0x07050301u))
                        : make_uint2(w[p][0], w[p][1]);
}

// kThreads, a wave or the workgroup, take rows_each neighbouring rows, which mostly belong to one expert, and keep that expert's scales and
// a row's products in registers; kPasses pieces per thread.  kWhole: the rows' pieces are whole.  One read of dy and one write of the
// digits: bound by HBM, and for a few thousand rows by the turns to memory that a row takes one after another.  4096 rows of 1408 of 8
// experts, bf16: 8.8 us with workgroups, 7.7 us with waves (3.0 TB/s); 2048 rows of 4096: 8.1 us (4.1 TB/s).
template <typename T, int kPlanes, int kThreads, int kPasses, bool kWhole>
__device__ __forceinline__ void digit_rows(const DigitArgs &A, int64_t block, int rows_each)
{
    const int thread = threadIdx.x % kThreads;
    const int64_t first = (block * (256 / kThreads) + threadIdx.x / kThreads) * rows_each;
    const int64_t end = first + rows_each < A.rows ? first + rows_each : A.rows;
    float ws[kPasses][8];
    int expert = -1;
    for (int64_t row = first; row < end; ++row) {
        const T *dy = (const T *)A.dy + row * A.ld_dy;
        Raw8 raw[kPasses];  // (asked for ahead of the expert, whose place takes two more turns to memory)
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int c = (p * kThreads + thread) * 8, at = c < A.n ? c : 0;
            raw[p] = kWhole ? load_whole_piece(dy + at) : load_piece(dy + at, A.n - c);
        }
        const int e = expert_of(A.offsets, A.experts, row);
        if (e < 0) continue;  // (the product does not look at it)
        if (e != expert) {
            expert = e;
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                const int c = (p * kThreads + thread) * 8;
                const int64_t at = (int64_t)e * A.n + (c < A.n ? c : 0);
                const int left = kWhole ? 8 : A.n - c;
                if (A.ws_f16)
                    unpack8(load_piece((const __half *)A.ws + at, left), ws[p], (const __half *)nullptr);
                else
                    unpack8(load_piece((const float *)A.ws + at, left), ws[p], (const float *)nullptr);
            }
        }
        float v[kPasses][8];
        uint32_t m = 0;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const bool in = (p * kThreads + thread) * 8 < A.n;
            unpack8(raw[p], v[p], (const T *)nullptr);
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                v[p][r] = in ? v[p][r] * ws[p][r] : 0.0f;
                const uint32_t b = __float_as_uint(v[p][r]) & 0x7FFFFFFFu;
                m = m > b ? m : b;
            }
        }
        const RowFactor f = row_factor<kPlanes>(max_over<kThreads>(m));
        if (thread == 0) A.factor[row] = f.factor;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int c = (p * kThreads + thread) * 8;
            if (c >= A.np) continue;
            uint2 d[kPlanes];
            digits8<kPlanes>(v[p], f, A.odd_last, d);
#pragma unroll
            for (int q = 0; q < kPlanes; ++q) *(uint2 *)(A.planes + ((int64_t)q * A.rows + row) * A.np + c) = d[q];
        }
    }
}

// Wider rows; the second look at a row comes from the caches.
template <typename T, int kPlanes>
__device__ __forceinline__ void digit_rows_wide(const DigitArgs &A, int64_t block, int rows_each)
{
    const int64_t end = (block + 1) * rows_each < A.rows ? (block + 1) * rows_each : A.rows;
    for (int64_t row = block * rows_each; row < end; ++row) {
        const int expert = expert_of(A.offsets, A.experts, row);
        if (expert < 0) continue;
        const T *dy = (const T *)A.dy + row * A.ld_dy;
        const int64_t s0 = (int64_t)expert * A.n;
        auto entry = [&](int c) { return c < A.n ? to_float(dy[c]) * load_scale(A.ws, s0 + c, A.ws_f16) : 0.0f; };
        uint32_t m = 0;
        for (int c = threadIdx.x; c < A.n; c += 256) {
            const uint32_t b = __float_as_uint(entry(c)) & 0x7FFFFFFFu;
            m = m > b ? m : b;
        }
        const RowFactor f = row_factor<kPlanes>(max_over<256>(m));
        if (threadIdx.x == 0) A.factor[row] = f.factor;
        for (int c = threadIdx.x * 8; c < A.np; c += 2048) {
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = entry(c + r);
            uint2 d[kPlanes];
            digits8<kPlanes>(v, f, A.odd_last, d);
#pragma unroll
            for (int q = 0; q < kPlanes; ++q) *(uint2 *)(A.planes + ((int64_t)q * A.rows + row) * A.np + c) = d[q];
        }
    }
}

struct TransposeArgs {
    const uint8_t *w;
    int8_t *out;  // [experts][k][np]
    const int32_t *offsets;
    int64_t ldw, w_step;
    int n, k, np;
};

__device__ __forceinline__ bool has_rows(const int32_t *offsets, int expert) { return !offsets || offsets[expert] < offsets[expert + 1]; }

constexpr int kTr = 128;

// 128 outputs x 128 inputs per workgroup, workgroup `block` of all.  A thread reads 16 codes of four neighbouring outputs, turns them in
// registers, 4 x 4 bytes at a time, and stores words of four outputs to LDS, from where the result's rows leave in whole lines.  Codes of 4
// and 2 bits come out as bytes with the code at the top, 16 or 64 times its value.  One read of w, one write: bound by HBM (4096 x 4096 bytes
// with the digits of 2048 bf16 rows: 13.5 us, 5.0 TB/s).
template <int kBits>
__device__ __forceinline__ void transpose_tile(const TransposeArgs &A, uint32_t block)
{
    constexpr int kLd = kTr / 4 + 1;
    __shared__ uint32_t s[kTr * kLd];
    const uint32_t across = (uint32_t)(A.k + kTr - 1) / kTr, down = (uint32_t)A.np / kTr;
    const int expert = (int)(block / (across * down));
    if (!has_rows(A.offsets, expert)) return;
    const int k0 = (int)(block % across) * kTr, o0 = (int)(block / across % down) * kTr;
    const int quad = threadIdx.x >> 3, part = (threadIdx.x & 7) * 16;
    uint32_t c[4][4] = {};  // [output][word]
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int o = o0 + quad * 4 + r;
        if (o >= A.n || k0 + part >= A.k) continue;
        const uint8_t *p = A.w + expert * A.w_step + (int64_t)o * A.ldw + (int64_t)(k0 + part) * kBits / 8;
        if constexpr (kBits == 8) {
            const uint4 v = *(const uint4 *)p;
            c[r][0] = v.x; c[r][1] = v.y; c[r][2] = v.z; c[r][3] = v.w;
        } else {
            uint32_t raw[kBits / 2];
#pragma unroll
            for (int j = 0; j < kBits / 2; ++j) raw[j] = ((const uint32_t *)p)[j];
            const i32x4 v = step_codes<kBits, true>(raw, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) c[r][j] = (uint32_t)v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t t0 = __builtin_amdgcn_perm(c[1][j], c[0][j], 0x05010400u), t1 = __builtin_amdgcn_perm(c[1][j], c[0][j], 0x07030602u);
        const uint32_t u0 = __builtin_amdgcn_perm(c[3][j], c[2][j], 0x05010400u), u1 = __builtin_amdgcn_perm(c[3][j], c[2][j], 0x07030602u);
        uint32_t *q = s + (part + 4 * j) * kLd + quad;
        q[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
        q[kLd] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
        q[2 * kLd] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
        q[3 * kLd] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 32 + quad, k = k0 + row;
        if (k >= A.k) continue;
        const uint32_t *q = s + row * kLd + part / 4;
        *(uint4 *)(A.out + ((int64_t)expert * A.k + k) * A.np + o0 + part) = make_uint4(q[0], q[1], q[2], q[3]);
    }
}

// Both in one launch: neither needs the other.  The first digit_blocks workgroups write digits (kPasses 0: of the widest rows), the others
// transpose (kBits 0: there are none).
template <typename T, int kPlanes, int kThreads, int kPasses, bool kWhole, int kBits>
__global__ __launch_bounds__(256) void linear_prepare_kernel(DigitArgs D, int rows_each, uint32_t digit_blocks, TransposeArgs R)
{
    if constexpr (kBits != 0) {
        if (blockIdx.x >= digit_blocks) {
            transpose_tile<kBits>(R, blockIdx.x - digit_blocks);
            return;
        }
    }
    if constexpr (kPasses == 0)
        digit_rows_wide<T, kPlanes>(D, blockIdx.x, rows_each);
    else
        digit_rows<T, kPlanes, kThreads, kPasses, kWhole>(D, blockIdx.x, rows_each);
}

// The same for any width and alignment, 64 x 64 codes one by one.
__global__ __launch_bounds__(256) void linear_transpose_any_kernel(TransposeArgs A, int bits)
{
    __shared__ __align__(16) uint8_t s[64][64 + 4];
    const int expert = blockIdx.z;
    if (!has_rows(A.offsets, expert)) return;
    const int k0 = blockIdx.x * 64, o0 = blockIdx.y * 64, per = 8 / bits;
    const int row = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;
    const uint8_t *w = A.w + expert * A.w_step + (int64_t)(o0 + row) * A.ldw;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const int k = k0 + part + j;
        s[row][part + j] = o0 + row < A.n && k < A.k ? (uint8_t)(w[k / per] << (8 - bits - (k % per) * bits)) & (0xFF00u >> bits) : 0;
    }
    __syncthreads();
    const int k = k0 + row;  // now a row of the result
    if (k >= A.k) return;
#pragma unroll
    for (int j = 0; j < 16; ++j) A.out[((int64_t)expert * A.k + k) * A.np + o0 + part + j] = (int8_t)s[part + j][row];
}

int padded(int n) { return (n + 127) / 128 * 128; }

template <typename T, int kPlanes, int kBits>
hipError_t launch_prepare(const DigitArgs &D, const TransposeArgs &R, uint32_t transpose_blocks, hipStream_t stream)
{
    auto launch = [&](auto THREADS, auto PASSES) {
        constexpr int threads = decltype(THREADS)::value, passes = decltype(PASSES)::value, at_once = 256 / threads;
        // beyond 16384 waves they take several rows each
        const int rows_each = (int)((D.rows + 4096 * at_once - 1) / (4096 * at_once));
        const int64_t per_block = (int64_t)rows_each * at_once;
        const uint32_t digit_blocks = (uint32_t)((D.rows + per_block - 1) / per_block);
        const dim3 grid(digit_blocks + transpose_blocks);
        if constexpr (passes != 0) {
            if (D.n % 8 == 0) {
                hipLaunchKernelGGL((linear_prepare_kernel<T, kPlanes, threads, passes, true, kBits>), grid, dim3(256), 0, stream, D, rows_each,
                                   digit_blocks, R);
                return hipGetLastError();
            }
        }
        hipLaunchKernelGGL((linear_prepare_kernel<T, kPlanes, threads, passes, false, kBits>), grid, dim3(256), 0, stream, D, rows_each, digit_blocks,
                           R);
        return hipGetLastError();
    };
    typedef std::integral_constant<int, 64> Wave;
    typedef std::integral_constant<int, 256> Workgroup;
    if (D.np > 16384) return launch(Workgroup{}, std::integral_constant<int, 0>{});
    if constexpr (kBits == 0) {
        // (beside transposing workgroups their registers cost more than the barrier of a workgroup's row)
        if (D.np <= 512) return launch(Wave{}, std::integral_constant<int, 1>{});
        if (D.np <= 2048) return launch(Wave{}, std::integral_constant<int, 4>{});
    } else {
        if (D.np <= 2048) return launch(Workgroup{}, std::integral_constant<int, 1>{});
    }
    if (D.np <= 4096) return launch(Workgroup{}, std::integral_constant<int, 2>{});
    if (D.np <= 8192) return launch(Workgroup{}, std::integral_constant<int, 4>{});
    return launch(Workgroup{}, std::integral_constant<int, 8>{});
}

// digits, and unless bits is 0 the weights
template <typename T, int kPlanes>
hipError_t prepare(const DigitArgs &D, const TransposeArgs &R, int bits, hipStream_t stream)
{
    if (bits == 0) return launch_prepare<T, kPlanes, 0>(D, R, 0, stream);
    const int64_t tiles = (int64_t)((R.k + kTr - 1) / kTr) * (R.np / kTr) * D.experts;
    if (R.k % 16 == 0 && (uintptr_t)R.w % (2 * bits) == 0 && R.ldw % (2 * bits) == 0 && tiles < (int64_t)1 << 23) {
        if (bits == 8) return launch_prepare<T, kPlanes, 8>(D, R, (uint32_t)tiles, stream);
        if (bits == 4) return launch_prepare<T, kPlanes, 4>(D, R, (uint32_t)tiles, stream);
        return launch_prepare<T, kPlanes, 2>(D, R, (uint32_t)tiles, stream);
    }
    const hipError_t e = launch_prepare<T, kPlanes, 0>(D, R, 0, stream);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((R.k + 63) / 64), (unsigned)(R.np / 64), (unsigned)D.experts);
    hipLaunchKernelGGL(linear_transpose_any_kernel, grid, dim3(256), 0, stream, R, bits);
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
    TransposeArgs R{};
    R.w = (const uint8_t *)w;
    R.out = (int8_t *)(base + L.weights);
    R.offsets = offsets;
    R.ldw = ldw;
    R.w_step = (int64_t)n * ldw;
    R.n = n;
    R.k = k;
    R.np = np;
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
    LinearArgs across = A;
    across.w = (const uint8_t *)w;
    across.ldw = ldw;
    across.w_step = R.w_step;
    across.w_rows = n;
    const bool as_they_are = linear_across_is_quicker(across, A, wbits, planes);
    const int turn = as_they_are ? 0 : wbits;
    D.odd_last = as_they_are && wbits < 8;
    const hipError_t e = dtype == BQ_F32   ? prepare<float, 3>(D, R, turn, stream)
                         : dtype == BQ_F16 ? prepare<__half, 2>(D, R, turn, stream)
                                           : prepare<bf16_t, 2>(D, R, turn, stream);
    if (e != hipSuccess) return e;
    if (as_they_are) return launch_linear_across(across, wbits, planes, stream);
    A.factor /= (float)(1 << (8 - wbits));
    return launch_linear(A, 8, 8, planes, stream);
}

}  // namespace bq
