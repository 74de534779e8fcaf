// The product for many rows: a workgroup takes a tile of tokens x channels and walks along the sum's index 128 codes at a time, through
// two stages in LDS.  The stages are filled by direct loads from memory (16 bytes per lane, no registers in between); one stage is
// loaded while the other is multiplied.
//
// LDS rows are the codes of 128 inputs (128, 64 or 32 bytes), rows of x and of w after one another.  A direct load writes its 64
// lanes' pieces in lane order, so the order of a row's 16-byte pieces is made by which piece a lane loads: piece ^ f(row), with f such
// that the 8 lanes of a 16-byte read that go together fall on different banks.
//
// A lane's 16 codes of the two matrix instructions of a stage are neighbours (32 g + 16 s .. of lane group g, step s): with packed codes
// one read then serves both.  Row i of the first operand's piece j is channel 16 (i / 4) + 4 j + i % 4 of the wave's 64: a lane ends
// with 16 consecutive channels of one token.
#pragma once

#include "bq_linear_codes.h"

namespace bq {

// Waves of a workgroup along tokens and channels, 16-row pieces of a wave along tokens (of x's rows: planes count); 64 channels per wave.
template <int kWavesT, int kWavesN, int kPieces>
struct TileShape {
    static constexpr int waves_t = kWavesT, waves_n = kWavesN, pieces = kPieces;
    static constexpr int waves = kWavesT * kWavesN, threads = 64 * waves;
    static constexpr int x_rows = kWavesT * kPieces * 16, w_rows = kWavesN * 64;
};

// f of the header comment; kPieceBytes: bytes of an LDS row.  x rows are read 16 in a row, w rows as i -> 16 (i / 4) + i % 4.
template <int kRowBytes>
__device__ __forceinline__ int x_turn(int row)
{
    return kRowBytes == 128 ? row & 7 : (row >> 1) & 3;
}
template <int kRowBytes>
__device__ __forceinline__ int w_turn(int row)
{
    return kRowBytes == 128 ? (row & 3) | ((row >> 2) & 4) : kRowBytes == 64 ? ((row >> 1) & 1) | ((row >> 3) & 2) : (row >> 4) & 1;
}

__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, const uint8_t *base)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" : : "v"(offset), "s"(lds), "s"(base) : "memory");
}

template <int kXBits, int kWBits, int kPlanes, typename Shape>
__global__ __launch_bounds__(Shape::threads, 1) void linear_tile_kernel(LinearArgs A)
{
    constexpr int kXRow = 16 * kXBits, kWRow = 16 * kWBits;  // bytes of 128 codes
    constexpr int kXBytes = Shape::x_rows * kXRow, kWBytes = Shape::w_rows * kWRow, kStage = kXBytes + kWBytes;
    constexpr int kXLoads = kXBytes / 1024 / Shape::waves, kWLoads = kWBytes / 1024 / Shape::waves;
    static_assert(kXLoads * 1024 * Shape::waves == kXBytes && kWLoads * 1024 * Shape::waves == kWBytes, "whole loads per wave");
    static_assert(Shape::pieces % kPlanes == 0 && (kPlanes == 1 || kXBits == 8), "planes of a token in one wave");
    constexpr int kTokens = Shape::x_rows / kPlanes, kP = Shape::pieces;
    constexpr bool kNatural = kXBits != kWBits;
    extern __shared__ __align__(16) uint8_t tile_lds[];

    // which tile: workgroups go round the 8 XCDs, each of which takes a contiguous eighth of the tiles; within it 8 tiles along the
    // tokens and then the next channels, so that what runs together shares its rows in the XCD's L2
    const int n_tiles = (A.n + Shape::w_rows - 1) / Shape::w_rows;
    const int64_t m_tiles = row_tiles(A, kTokens);
    const int64_t all = m_tiles * n_tiles, each = (all + 7) / 8;
    const int64_t idx = blockIdx.x >> 3;
    const int64_t tile = (int64_t)(blockIdx.x & 7) * each + idx;
    if (idx >= each || tile >= all) return;
    const int64_t band = tile / (8 * n_tiles), in_band = tile - band * (8 * n_tiles);
    const int64_t band_rows = m_tiles - band * 8 < 8 ? m_tiles - band * 8 : 8;
    RowTile rt = row_tile(A, band * 8 + in_band % band_rows, kTokens);
    rt = RowTile{__builtin_amdgcn_readfirstlane(rt.expert), uniform(rt.row0), uniform(rt.row_end)};
    const int o0 = (int)(in_band / band_rows) * Shape::w_rows;
    if (rt.row0 >= rt.row_end) return;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_t = wave / Shape::waves_n, wave_n = wave % Shape::waves_n;
    const int r16 = lane & 15, g = lane >> 4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)tile_lds;

    // loads: instruction q of the stage covers 1024 bytes of LDS, 8, 16 or 32 rows
    const uint8_t *x_base[kXLoads], *w_base;
    uint32_t x_off[kXLoads], w_off[kWLoads];
    int x_piece[kXLoads], w_piece[kWLoads];
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
        const int q = i * Shape::waves + wave, row = q * (1024 / kXRow) + lane / (kXRow / 16);
        const int plane = kPlanes == 1 ? 0 : (q * (1024 / kXRow) / 16) % kPlanes;
        const int token = kPlanes == 1 ? row : (row / (16 * kPlanes)) * 16 + row % 16;
        const int last = (int)(rt.row_end - rt.row0) - 1;
        x_piece[i] = (lane % (kXRow / 16)) ^ x_turn<kXRow>(row);
        x_base[i] = A.x + plane * A.plane_step + rt.row0 * A.ldx;
        x_off[i] = (uint32_t)(token < last ? token : last) * (uint32_t)A.ldx + x_piece[i] * 16;
    }
    w_base = A.w + rt.expert * A.w_step + (int64_t)o0 * A.ldw;
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
        const int row = (i * Shape::waves + wave) * (1024 / kWRow) + lane / (kWRow / 16);
        const int last = A.n - o0 - 1;
        w_piece[i] = (lane % (kWRow / 16)) ^ w_turn<kWRow>(row);
        w_off[i] = (uint32_t)(row < last ? row : last) * (uint32_t)A.ldw + w_piece[i] * 16;
    }
    const int stages = (A.k + 127) / 128;
    const int x_tail = (int)((int64_t)A.k * kXBits / 128) % (kXRow / 16), w_tail = (int)((int64_t)A.k * kWBits / 128) % (kWRow / 16);  // pieces of the last stage
    auto load_stage = [&](int s) {
        const uint32_t at = lds0 + (s & 1) * kStage + wave * 1024;
        const bool short_x = x_tail && s == stages - 1, short_w = w_tail && s == stages - 1;  // its missing pieces: any other one
#pragma unroll
        for (int i = 0; i < kXLoads; ++i)
            load_to_lds(at + i * Shape::waves * 1024, short_x && x_piece[i] >= x_tail ? x_off[i] - x_piece[i] * 16 : x_off[i], x_base[i] + (int64_t)s * kXRow);
#pragma unroll
        for (int i = 0; i < kWLoads; ++i)
            load_to_lds(at + kXBytes + i * Shape::waves * 1024, short_w && w_piece[i] >= w_tail ? w_off[i] - w_piece[i] * 16 : w_off[i],
                        w_base + (int64_t)s * kWRow);
    };

    // reads
    const int x_row = wave_t * kP * 16 + r16, w_row = wave_n * 64 + 16 * (r16 >> 2) + (r16 & 3);
    i32x4 acc[kP][4] = {};
    load_stage(0);
    for (int s = 0; s < stages; ++s) {
        // this wave's loads of stage s have landed, and with the barrier everyone's; everyone has read the other stage
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < stages) load_stage(s + 1);
        uint8_t *xl = tile_lds + (s & 1) * kStage;
        const uint8_t *wl = xl + kXBytes;
        if (x_tail && s == stages - 1) {  // codes behind the last input count as 0 (then the weights' do not matter)
            for (int p = threadIdx.x; p < Shape::x_rows * (kXRow / 16); p += Shape::threads) {
                const int row = p / (kXRow / 16), at = p % (kXRow / 16);
                if ((at ^ x_turn<kXRow>(row)) >= x_tail) *(uint4 *)(xl + row * kXRow + at * 16) = make_uint4(0, 0, 0, 0);
            }
            __syncthreads();
        }
        uint32_t wv[4][kWBits == 2 ? 2 : kWBits == 4 ? 4 : 8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = w_row + 4 * j;
            if constexpr (kWBits == 2) {
                const uint2 v = *(const uint2 *)(wl + row * kWRow + ((g >> 1) ^ w_turn<kWRow>(row)) * 16 + (g & 1) * 8);
                wv[j][0] = v.x; wv[j][1] = v.y;
            } else {
#pragma unroll
                for (int h = 0; h < (kWBits == 8 ? 2 : 1); ++h) {
                    const uint4 v = *(const uint4 *)(wl + row * kWRow + (((kWBits == 8 ? 2 * g : g) + h) ^ w_turn<kWRow>(row)) * 16);
                    wv[j][4 * h] = v.x; wv[j][4 * h + 1] = v.y; wv[j][4 * h + 2] = v.z; wv[j][4 * h + 3] = v.w;
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 a[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = step_codes<kWBits, kNatural>(wv[j], h);
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                const int row = x_row + 16 * i;
                i32x4 b;
                if constexpr (kXBits == 8) {
                    b = *(const i32x4 *)(xl + row * kXRow + ((2 * g + h) ^ x_turn<kXRow>(row)) * 16);
                } else {
                    const uint2 v = *(const uint2 *)(xl + row * kXRow + (g ^ x_turn<kXRow>(row)) * 16 + h * 8);
                    const uint32_t q[2] = {v.x, v.y};
                    b = step_codes<4, kNatural>(q, 0);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], b, acc[i][j], 0, 0, 0);
            }
        }
    }

    const int o = o0 + wave_n * 64 + g * 16;
    if (o >= A.n) return;
    float ws[16], bias[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const int64_t at = (int64_t)rt.expert * A.n + (o + c < A.n ? o + c : A.n - 1);
        ws[c] = A.ws ? load_scale(A.ws, at, A.ws_f16) : 1.0f;
        bias[c] = A.bias ? load_row_value(A.bias, at, A.dtype) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kP / kPlanes; ++i) {
        const int64_t t = rt.row0 + (wave_t * (kP / kPlanes) + i) * 16 + r16;
        if (t >= rt.row_end) continue;
        const float xs = load_scale(A.xs, t, A.xs_f16) * A.factor;
        float v[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            int part[kPlanes];
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) part[p] = acc[i * kPlanes + p][c >> 2][c & 3];
            v[c] = joined<kPlanes>(part) * xs;
            if (A.ws) v[c] *= ws[c];
            if (A.bias) v[c] += bias[c];
        }
        store_results<16>(A, t * A.ldy + o, v, A.n - o, A.y_quads);
    }
}

template <int kXBits, int kWBits, int kPlanes, typename Shape>
hipError_t launch_tile(const LinearArgs &A, hipStream_t stream)
{
    constexpr size_t kLds = 2 * (size_t)(Shape::x_rows * 16 * kXBits + Shape::w_rows * 16 * kWBits);
    static LdsLimitOnce limit;
    const hipError_t e = limit.set((const void *)linear_tile_kernel<kXBits, kWBits, kPlanes, Shape>, kLds);
    if (e != hipSuccess) return e;
    const int64_t n_tiles = (A.n + Shape::w_rows - 1) / Shape::w_rows;
    const int64_t all = row_tiles_bound(A, Shape::x_rows / kPlanes) * n_tiles;
    hipLaunchKernelGGL((linear_tile_kernel<kXBits, kWBits, kPlanes, Shape>), dim3((unsigned)((all + 7) / 8 * 8)), dim3(Shape::threads), kLds,
                       stream, A);
    return hipGetLastError();
}

typedef TileShape<2, 4, 8> TileLarge;   // 256 tokens x 256 channels, or 128 x 256 of two planes
typedef TileShape<2, 4, 6> TileLarge3;  // 64 tokens of three planes x 256
typedef TileShape<2, 2, 4> TileSmall;   // 128 x 128, or 64 x 128 of two planes
typedef TileShape<2, 2, 6> TileSmall3;  // 64 tokens of three planes x 128

}  // namespace bq
