// The product for few rows.  A workgroup takes kBlocks x kCols pieces of 16 tokens x 16 channels; its waves share the sum's index, step by
// step, so that the workgroup reads its channels' codes front to back, every code once, and every wave works for itself: it loads
// the codes of its steps into a ring of its own in LDS (directly, 16 bytes per lane, whole lines: in the order the matrix instruction
// wants them a load touched 64 lines instead of 8 or 16, and the address units were what bound the kernel: 33 KB/us and compute unit),
// reads them from there and multiplies, with no barrier.  The waves' partial sums are joined through LDS, integers in whatever order, a
// gradient's float32 sums wave after wave.  Decoding (a few tokens, kCols = 1) is bound by the weights' bytes; with more tokens the pieces grow, since a code of x
// is read once per kCols pieces and one of w once per kBlocks, and the bound is what a compute unit gets from L2, 87 KB/us of
// direct loads alone, and the 3 to 4 us of start, first loads and joining.  One token, 8-bit
// codes 4096 -> 4096: 4.6 us, 3.6 TB/s; 37 tokens, 4-bit weights 11008 -> 4096: 10.2 us, 2.2 TB/s of weights, each read twice.
#pragma once

#include "bq_linear_codes.h"

namespace bq {

template <int kXBits, int kWBits, int kTerms, int kBlocks, int kCols, bool kWide>
__global__ __launch_bounds__((64 * RowsShape<kXBits, kWBits, kTerms, kBlocks, kCols, kWide>::waves),
                             (RowsShape<kXBits, kWBits, kTerms, kBlocks, kCols, kWide>::per_simd)) void linear_rows_kernel(LinearArgs A)
{
    typedef RowsShape<kXBits, kWBits, kTerms, kBlocks, kCols, kWide> S;
    constexpr int kFrags = S::frags, kWaves = S::waves, kDepth = S::depth, kPairs = S::pairs, kChunk = S::chunk;
    constexpr int kXSub = S::x_row == 256 ? 2 : 1, kXLine = S::x_row / kXSub;  // rows of 256 bytes lie as two of 128
    constexpr int kXWords = S::x_row / 16, kWWords = S::w_row / 16;            // of a lane: a quarter of a row
    constexpr int kXLoads = S::x_bytes / 1024, kWLoads = S::w_bytes / 1024, kLoads = kXLoads + kWLoads;
    constexpr bool kFloat = kXBits == 16, kNatural = kXBits != kWBits;
    static_assert(kFloat == (kTerms > 1) && (!kFloat || kWBits == 8), "codes, or a gradient");
    typedef typename SumType<kFloat>::type Sum;
    extern __shared__ __align__(16) uint8_t rows_lds[];
    Sum(*const s_part)[kChunk][64] = (Sum(*)[kChunk][64])rows_lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16 * kCols;
    const int expert = A.offsets ? blockIdx.z : 0;
    int64_t row_a, row_b;
    expert_rows(A, expert, &row_a, &row_b);
    uint8_t *const ring = rows_lds + wave * (kDepth * S::step);
    const uint32_t ring0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)rows_lds + wave * (kDepth * S::step);

    // what this lane loads of a step: instruction i of w covers 1024 / w_row channels
    const uint8_t *const w_base = A.w + expert * A.w_step + (int64_t)o0 * A.ldw;
    uint32_t w_off[kWLoads];
    int w_piece[kWLoads];
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
        const int row = i * (1024 / S::w_row) + lane / (S::w_row / 16), last = A.n - o0 - 1;
        w_piece[i] = (lane % (S::w_row / 16)) ^ lds_turn<S::w_row, kWWords / 4>(row & 15);
        w_off[i] = (uint32_t)(row < last ? row : last) * (uint32_t)A.ldw;
    }
    const int steps = (A.k + S::codes - 1) / S::codes;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;
    // 16-byte pieces of the last step, where it is short
    const int x_tail = (int)((int64_t)A.k * kXBits / 128) % (S::x_row / 16), w_tail = (int)((int64_t)A.k * kWBits / 128) % (S::w_row / 16);
    const int64_t pass = 16 * kBlocks;
    for (int64_t row0 = row_a + blockIdx.y * pass; row0 < row_b; row0 += gridDim.y * pass) {
        const uint8_t *x_base[kXLoads];
        uint32_t x_off[kXLoads];
        int x_piece[kXLoads];
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            // x lies as [half of a row][plane and 16 tokens][token]
            const int line = i * (1024 / kXLine) + lane / (kXLine / 16), half = i * (1024 / kXLine) / (16 * kFrags);
            const int frag = i * (1024 / kXLine) / 16 % kFrags, token = 16 * (frag / kTerms) + line % 16;
            const int last = (int)(row_b - row0 < pass ? row_b - row0 : pass) - 1;
            x_piece[i] = half * 8 + ((lane % (kXLine / 16)) ^ lds_turn<kXLine, kXWords / 4>(line & 15));
            x_base[i] = A.x + (frag % kTerms) * A.plane_step + row0 * A.ldx;
            x_off[i] = (uint32_t)(token < last ? token : last) * (uint32_t)A.ldx;
        }
        auto load = [&](int i, int place) {  // the wave's i-th step
            const int s = wave + i * kWaves;
            const bool last = s == steps - 1;  // a piece behind the last input: the step's first one
#pragma unroll
            for (int n = 0; n < kXLoads; ++n)
                load_to_lds(ring0 + place * S::step + n * 1024, x_off[n] + (last && x_tail && x_piece[n] >= x_tail ? 0 : x_piece[n]) * 16,
                            x_base[n] + (int64_t)s * S::x_row);
#pragma unroll
            for (int n = 0; n < kWLoads; ++n)
                load_to_lds(ring0 + place * S::step + S::x_bytes + n * 1024,
                            w_off[n] + (last && w_tail && w_piece[n] >= w_tail ? 0 : w_piece[n]) * 16, w_base + (int64_t)s * S::w_row);
        };
        constexpr int kSums = kFloat ? 2 * kBlocks : kBlocks;  // (first terms, others)
        Sum acc[kCols][kSums] = {};
        if (row0 != row_a + blockIdx.y * pass) __syncthreads();  // the pass before has read its sums
        for (int i = 0; i < kDepth && i < mine; ++i) load(i, i);
        for (int i = 0, place = 0; i < mine; ++i) {
            if (i + kDepth <= mine)
                asm volatile("s_waitcnt vmcnt(%0)" : : "n"((kDepth - 1) * kLoads) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            uint32_t wv[kCols][kWWords], xv[kFrags][kXWords];
            const uint8_t *const at = ring + place * S::step;
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
#pragma unroll
                for (int j = 0; j < kXWords / 4; ++j) {
                    const int piece = g * (kXWords / 4) + j;
                    const uint4 q = *(const uint4 *)(at + ((piece / (kXLine / 16)) * kFrags * 16 + f * 16 + r16) * kXLine +
                                                     ((piece % (kXLine / 16)) ^ lds_turn<kXLine, kXWords / 4>(r16)) * 16);
                    xv[f][4 * j] = q.x; xv[f][4 * j + 1] = q.y; xv[f][4 * j + 2] = q.z; xv[f][4 * j + 3] = q.w;
                }
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int j = 0; j < kWWords / 4; ++j) {
                    const uint4 q = *(const uint4 *)(at + S::x_bytes + (c * 16 + r16) * S::w_row +
                                                     ((g * (kWWords / 4) + j) ^ lds_turn<S::w_row, kWWords / 4>(r16)) * 16);
                    wv[c][4 * j] = q.x; wv[c][4 * j + 1] = q.y; wv[c][4 * j + 2] = q.z; wv[c][4 * j + 3] = q.w;
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read: the place may be loaded again
            if (i + kDepth < mine) load(i + kDepth, place);
            place = place + 1 == kDepth ? 0 : place + 1;
            if (x_tail && wave + i * kWaves == steps - 1) {  // codes behind the last input count as 0
#pragma unroll
                for (int f = 0; f < kFrags; ++f)
#pragma unroll
                    for (int j = 0; j < kXWords; ++j)
                        if (g * (kXWords / 4) + j / 4 >= x_tail) xv[f][j] = 0;
            }
#pragma unroll
            for (int s = 0; s < S::codes / (kFloat ? 32 : 64); ++s) {
                i32x4 a[kCols];
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    if constexpr (kFloat)
                        a[c] = half_codes8(wv[c][2 * s], wv[c][2 * s + 1]);
                    else
                        a[c] = step_codes<kWBits, kNatural>(wv[c], s);
                }
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    const i32x4 b = step_codes<kFloat ? 8 : kXBits, kNatural>(xv[f], s);  // (terms lie as 16 bytes of a step, too)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) {
                        Sum &sum = acc[c][kFloat ? f / kTerms * 2 + (f % kTerms != 0) : f];
                        sum = multiply(a[c], b, sum);
                    }
                }
            }
        }
#pragma unroll
        for (int first = 0; first < kPairs; first += kChunk) {
            __syncthreads();  // (the codes, or the sums before, have been read)
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                if (first + i >= kPairs) continue;
                const Sum *const piece = acc[(first + i) / kBlocks];
                const int b = (first + i) % kBlocks;
                if constexpr (kFloat) {
                    Sum v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = terms_sum(piece[2 * b][r], piece[2 * b + 1][r]);
                    s_part[wave][i][lane] = v;
                } else {
                    s_part[wave][i][lane] = piece[b];
                }
            }
            __syncthreads();
            const int pair = first + wave, block = pair % kBlocks, col = pair / kBlocks;
            if (wave >= kChunk || pair >= kPairs) continue;
            Sum sum = s_part[0][wave][lane];
#pragma unroll
            for (int v = 1; v < kWaves; ++v) sum += s_part[v][wave][lane];
            const int64_t t = row0 + 16 * block + r16;
            const int o = o0 + 16 * col + 4 * g;
            if (t >= row_b || o >= A.n) continue;
            float v[4];
            if constexpr (kFloat) {
                const int exponent = ((const int *)A.xs)[t];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = ldexpf(sum[r] * A.factor, exponent);
            } else {
                const float xs = load_scale(A.xs, t, A.xs_f16);
                int64_t at[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) at[r] = (int64_t)expert * A.n + (o + r < A.n ? o + r : A.n - 1);
                float ws[4], bias[4];
                load_scales(A.ws, A.ws_f16, at, ws);
                channel_bias(A, at, bias);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    v[r] = scaled(sum[r], A.factor, xs, ws[r]);
                    if (A.bias) v[r] += bias[r];
                }
            }
            store_results<4>(A, t * A.ldy + o, v, A.n - o);
        }
    }
}

template <int kXBits, int kWBits, int kTerms, int kBlocks, int kCols, bool kWide>
hipError_t launch_rows_shape(const LinearArgs &A, dim3 grid, hipStream_t stream)
{
    typedef RowsShape<kXBits, kWBits, kTerms, kBlocks, kCols, kWide> S;
    static LdsLimitOnce limit;
    const hipError_t e = limit.set((const void *)linear_rows_kernel<kXBits, kWBits, kTerms, kBlocks, kCols, kWide>, S::lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((linear_rows_kernel<kXBits, kWBits, kTerms, kBlocks, kCols, kWide>), grid, dim3(64 * S::waves), S::lds, stream, A);
    return hipGetLastError();
}

template <int kXBits, int kWBits, int kTerms, int kBlocks, int kCols>
hipError_t launch_rows(const LinearArgs &A, hipStream_t stream)
{
    const RowsGrid g = rows_grid(size_of(A), kBlocks, kCols);
    const dim3 grid((unsigned)g.along_channels, (unsigned)g.along_rows, (unsigned)g.experts);
    constexpr bool kPair = RowsShape<kXBits, kWBits, kTerms, kBlocks, kCols, false>::exists;
    if constexpr (kPair) {
        if (kWBits < 8 || !rows_alone(g)) return launch_rows_shape<kXBits, kWBits, kTerms, kBlocks, kCols, false>(A, grid, stream);
    }
    if constexpr (!kPair || kWBits == 8) {
        static_assert(RowsShape<kXBits, kWBits, kTerms, kBlocks, kCols, true>::exists, "fits the LDS");
        return launch_rows_shape<kXBits, kWBits, kTerms, kBlocks, kCols, true>(A, grid, stream);
    }
}

// blocks x cols: 1x1, 1x2, 1x4, 2x1, 2x2, 4x2; of a gradient's terms 1x1, 1x2, 2x1 and (two terms) 2x2
template <int kXBits, int kWBits, int kTerms>
hipError_t launch_rows_of(const LinearArgs &A, int blocks, int cols, hipStream_t stream)
{
    if constexpr (kTerms == 1) {
        if (blocks == 4) return launch_rows<kXBits, kWBits, 1, 4, 2>(A, stream);
        if (cols == 4) return launch_rows<kXBits, kWBits, 1, 1, 4>(A, stream);
    }
    if constexpr (kTerms < 3) {
        if (blocks == 2 && cols == 2) return launch_rows<kXBits, kWBits, kTerms, 2, 2>(A, stream);
    }
    if (blocks == 2) return launch_rows<kXBits, kWBits, kTerms, 2, 1>(A, stream);
    return cols == 2 ? launch_rows<kXBits, kWBits, kTerms, 1, 2>(A, stream) : launch_rows<kXBits, kWBits, kTerms, 1, 1>(A, stream);
}

}  // namespace bq
