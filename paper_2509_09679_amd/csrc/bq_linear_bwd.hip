// What the gradient of a quantised product needs in front of the product itself: dy times the weights' scales as sums of binary16 numbers,
// and, where the product does not read them as they lie, the weights' codes transposed, both with the summed index (the layer's outputs)
// contiguous and padded with zeros.
//
// Terms.  v = dy ws, a float32 number, times the power of two that brings the row's largest into [2^14, 2^15), is written as
// h + 2^-11 (m + l), each the binary16 number nearest to what those before it leave: 22 bits of v with h and m (16-bit rows), 33 with
// all three (float32 rows, so none of v's 24 is lost), whatever the row's other entries are.  What binary16's smallest number cuts off is
// 2^-50 of the row's largest.  (Fixed-point digits relative to the row's largest entry, multiplied in integers, are half the
// matrix cores' work, but lose the small entries of a row: of a softmax's gradient most of the sum.)  Two terms and not three for 16-bit
// rows: the rounding of the result is 2^-12 or 2^-9, and three take half as long again.  The sums are float32, of the products with h and
// of the others apart, so that only the former's roundings, one per 32 products, count; products of binary16 numbers are exact.  A row with
// an infinity or a NaN has NaN in m: its gradient is NaN throughout.
#include <type_traits>

#include "bq_linear_codes.h"
#include "bq_piece.h"

namespace bq {

namespace {

struct TermArgs {
    const void *dy, *ws;
    _Float16 *planes;  // [kTerms][rows][np]
    int32_t *exponent; // [rows]: the terms are 2^-exponent times v
    const int32_t *offsets;
    int64_t rows, ld_dy;
    int n, np, experts, ws_f16;
    int spread;  // eight terms lie as 0, 4, 1, 5, 2, 6, 3, 7: how packed codes come out of a word with the fewest steps
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

// what a row's entries are divided by, as a power of two, from the bit pattern of its largest magnitude
__device__ __forceinline__ int row_exponent(uint32_t amax_bits)
{
    const float amax = __uint_as_float(amax_bits);
    // (v_frexp_exp gives 0 for 0, infinities and NaN)
    return amax_bits == 0 ? 0 : __builtin_amdgcn_frexp_expf(amax) - 15;
}

// The terms of 8 entries, by plane.
template <int kTerms>
__device__ __forceinline__ void terms8(const float (&v)[8], int exponent, int spread, uint4 (&t)[kTerms])
{
    float left[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int from = r == 0 || r == 7 ? r : r % 2 ? (r + 7) / 2 : r / 2;  // 0, 4, 1, 5, 2, 6, 3, 7
        left[r] = ldexpf(spread ? v[from] : v[r], -exponent);
    }
#pragma unroll
    for (int p = 0; p < kTerms; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = f32x2_to_f16x2_bits(left[2 * j], left[2 * j + 1]);
            const f16x2 h = __builtin_bit_cast(f16x2, w[j]);
#pragma unroll
            for (int r = 0; r < 2; ++r) left[2 * j + r] = (left[2 * j + r] - (float)h[r]) * (p == 0 ? kLowerTerms : 1.0f);
        }
        t[p] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int kTerms>
__device__ __forceinline__ void store_terms(const TermArgs &A, int64_t row, int c, const uint4 (&t)[kTerms])
{
#pragma unroll
    for (int p = 0; p < kTerms; ++p) *(uint4 *)(A.planes + ((int64_t)p * A.rows + row) * A.np + c) = t[p];
}

// kThreads, a wave or the workgroup, take rows_each neighbouring rows, which mostly belong to one expert, and keep that expert's scales and
// a row's products in registers; kPasses pieces per thread.  kWhole: the rows' pieces are whole.  One read of dy and one write of the
// terms: bound by HBM, and for a few thousand rows by the turns to memory that a row takes one after another.  bf16, 4096 rows of 1408
// of 8 experts: 8.4 us (4.1 TB/s); 2048 rows of 4096: 9 us (5.6 TB/s).
template <typename T, int kTerms, int kThreads, int kPasses, bool kWhole>
__device__ __forceinline__ void term_rows(const TermArgs &A, int64_t block, int rows_each)
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
        const int exponent = row_exponent(max_over<kThreads>(m));
        if (thread == 0) A.exponent[row] = exponent;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const int c = (p * kThreads + thread) * 8;
            if (c >= A.np) continue;
            uint4 t[kTerms];
            terms8<kTerms>(v[p], exponent, A.spread, t);
            store_terms<kTerms>(A, row, c, t);
        }
    }
}

// Wider rows; the second look at a row comes from the caches.
template <typename T, int kTerms>
__device__ __forceinline__ void term_rows_wide(const TermArgs &A, int64_t block, int rows_each)
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
        const int exponent = row_exponent(max_over<256>(m));
        if (threadIdx.x == 0) A.exponent[row] = exponent;
        for (int c = threadIdx.x * 8; c < A.np; c += 2048) {
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = entry(c + r);
            uint4 t[kTerms];
            terms8<kTerms>(v, exponent, A.spread, t);
            store_terms<kTerms>(A, row, c, t);
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
// beside the terms of 8 rows: 7.8 us, 4.3 TB/s).
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

// Both in one launch: neither needs the other.  The first term_blocks workgroups write terms (kPasses 0: of the widest rows), the others
// transpose (kBits 0: there are none).
template <typename T, int kTerms, int kThreads, int kPasses, bool kWhole, int kBits>
__global__ __launch_bounds__(256) void linear_prepare_kernel(TermArgs D, int rows_each, uint32_t term_blocks, TransposeArgs R)
{
    if constexpr (kBits != 0) {
        if (blockIdx.x >= term_blocks) {
            transpose_tile<kBits>(R, blockIdx.x - term_blocks);
            return;
        }
    }
    if constexpr (kPasses == 0)
        term_rows_wide<T, kTerms>(D, blockIdx.x, rows_each);
    else
        term_rows<T, kTerms, kThreads, kPasses, kWhole>(D, blockIdx.x, rows_each);
}

// The transposition for any width and alignment, 64 x 64 codes one by one.
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

int padded(int n) { return (n + 127) / 128 * 128; }  // rows' strides; the products sum over whole stages of 64

template <typename T, int kTerms, int kBits>
hipError_t launch_prepare(const TermArgs &D, const TransposeArgs &R, uint32_t transpose_blocks, hipStream_t stream)
{
    auto launch = [&](auto THREADS, auto PASSES) {
        constexpr int threads = decltype(THREADS)::value, passes = decltype(PASSES)::value, at_once = 256 / threads;
        // beyond 16384 waves they take several rows each
        const int rows_each = (int)((D.rows + 4096 * at_once - 1) / (4096 * at_once));
        const int64_t per_block = (int64_t)rows_each * at_once;
        const uint32_t term_blocks = (uint32_t)((D.rows + per_block - 1) / per_block);
        const dim3 grid(term_blocks + transpose_blocks);
        if constexpr (passes != 0) {
            if (D.n % 8 == 0) {
                hipLaunchKernelGGL((linear_prepare_kernel<T, kTerms, threads, passes, true, kBits>), grid, dim3(256), 0, stream, D, rows_each,
                                   term_blocks, R);
                return hipGetLastError();
            }
        }
        hipLaunchKernelGGL((linear_prepare_kernel<T, kTerms, threads, passes, false, kBits>), grid, dim3(256), 0, stream, D, rows_each, term_blocks,
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

// terms, and unless bits is 0 the weights
template <typename T, int kTerms>
hipError_t prepare(const TermArgs &D, const TransposeArgs &R, int bits, hipStream_t stream)
{
    if (bits == 0) return launch_prepare<T, kTerms, 0>(D, R, 0, stream);
    const int64_t tiles = (int64_t)((R.k + kTr - 1) / kTr) * (R.np / kTr) * D.experts;
    if (R.k % 16 == 0 && (uintptr_t)R.w % (2 * bits) == 0 && R.ldw % (2 * bits) == 0 && tiles < (int64_t)1 << 23) {
        if (bits == 8) return launch_prepare<T, kTerms, 8>(D, R, (uint32_t)tiles, stream);
        if (bits == 4) return launch_prepare<T, kTerms, 4>(D, R, (uint32_t)tiles, stream);
        return launch_prepare<T, kTerms, 2>(D, R, (uint32_t)tiles, stream);
    }
    const hipError_t e = launch_prepare<T, kTerms, 0>(D, R, 0, stream);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((R.k + 63) / 64), (unsigned)(R.np / 64), (unsigned)D.experts);
    hipLaunchKernelGGL(linear_transpose_any_kernel, grid, dim3(256), 0, stream, R, bits);
    return hipGetLastError();
}

}  // namespace

int linear_terms(int dtype) { return dtype == BQ_F32 ? 3 : 2; }

LinearBwdLayout linear_bwd_layout(int64_t rows, int n, int k, int experts, int dtype)
{
    LinearBwdLayout L;
    const size_t np = (size_t)padded(n);
    L.exponent = 0;
    L.planes = align256((size_t)rows * sizeof(int32_t));
    L.weights = L.planes + align256((size_t)linear_terms(dtype) * (size_t)rows * np * sizeof(_Float16));
    L.total = L.weights + align256((size_t)experts * (size_t)k * np);
    return L;
}

hipError_t launch_linear_bwd(const void *dy, int64_t ld_dy, const void *w, int wbits, int64_t ldw, const void *ws, int ws_f16,
                             const int32_t *offsets, void *dx, int64_t ld_dx, void *workspace, int64_t rows, int n, int k, int experts,
                             int dtype, hipStream_t stream)
{
    const LinearBwdLayout L = linear_bwd_layout(rows, n, k, experts, dtype);
    char *base = (char *)workspace;
    const int np = padded(n), terms = linear_terms(dtype);
    TermArgs D{};
    D.dy = dy;
    D.ws = ws;
    D.planes = (_Float16 *)(base + L.planes);
    D.exponent = (int32_t *)(base + L.exponent);
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
    A.xs = base + L.exponent;
    A.y = dx;
    A.offsets = offsets;
    A.rows = rows;
    A.ldx = np * (int64_t)sizeof(_Float16);
    A.ldw = np;
    A.ldy = ld_dx;
    A.w_step = (int64_t)k * np;
    A.plane_step = rows * A.ldx;
    A.k = (n + 63) / 64 * 64;
    A.n = k;
    A.experts = experts;
    A.dtype = dtype;
    A.factor = 1.0f;
    LinearArgs across = A;
    across.w = (const uint8_t *)w;
    across.ldw = ldw;
    across.w_step = R.w_step;
    across.w_rows = n;
    const bool as_they_are = linear_across_is_quicker(across, wbits, terms);
    const int turn = as_they_are ? 0 : wbits;
    D.spread = as_they_are && wbits < 8;
    const hipError_t e = dtype == BQ_F32   ? prepare<float, 3>(D, R, turn, stream)
                         : dtype == BQ_F16 ? prepare<__half, 2>(D, R, turn, stream)
                                           : prepare<bf16_t, 2>(D, R, turn, stream);
    if (e != hipSuccess) return e;
    if (as_they_are) return launch_linear_across(across, wbits, terms, stream);
    A.factor /= (float)(1 << (8 - wbits));
    return launch_linear_terms(A, terms, stream);
}

}  // namespace bq
