// The product for many rows: a workgroup takes a tile of tokens x channels and walks along the sum's index, 128 codes at a time, through a
// ring of stages in LDS.  The stages are filled by direct loads from memory (16 bytes per lane, no registers in between); one stage is
// multiplied while the others are loaded.
//
// LDS rows are the codes of a stage (128 bytes, 64 or 32 of packed codes), rows of x and of w after one another.  A direct load writes its 64
// lanes' pieces in lane order, so the order of a row's 16-byte pieces is made by which piece a lane loads: piece ^ f(row), with f such
// that the lanes of a read that go together fall on different banks.  (All but the reads of packed weights that lie across: across_turn.)
//
// Where a stage feeds two matrix instructions, a lane's 16 codes of the two are neighbours (32 g + 16 s .. of lane group g, step s):
// with packed codes one read then serves both.  Row i of the first operand's piece j is channel 16 (i / 4) + 4 j + i % 4 of the wave's 64:
// a lane ends with 16 consecutive channels of one token.
//
// Bound by the matrix cores (60 .. 66 % busy where the rounds of tiles are full, 47 .. 55 % where the last one is not or tiles are small) at the
// clock that the power limit leaves them, by what part of the last round is full, and with packed codes by the vector instructions that unpack
// them, 2.6 per matrix instruction.  4-bit codes, 16384 tokens, 8192 -> 8192: 735 .. 770 us, 2.9 POP/s, where a loop of the same instruction on
// random registers reaches 4.2; 8-bit codes, 1777 tokens, 4096 -> 11008: 80 .. 84 us, 2.0 POP/s; a gradient's two terms, 2048 tokens, 4096 -> 4096:
// 104 .. 115 us, 1.2 .. 1.3 PFLOP/s of binary16, where a loop of the same instruction on random registers reaches 1.96.
#pragma once

#include <type_traits>

#include "bq_linear_codes.h"

namespace bq {

// f of the header comment for w's rows, which are read as i -> 16 (i / 4) + i % 4; x's: lds_turn
template <int kRowBytes>
__device__ __forceinline__ int w_turn(int row)
{
    return kRowBytes == 128 ? ((row >> 1) & 1) | ((row >> 3) & 4) : kRowBytes == 64 ? (row >> 4) & 2 : (row >> 4) & 1;
}

// f for weights that lie across, rows of kRowBytes: a transposing read takes 8 bytes per lane, 32 lanes at a time, of 16 neighbouring
// bytes of 8 rows (8 bits) or 8 of 16 rows (4 and 2 bits) from either of two places 16 rows apart.  (The latter read every bank twice, a
// fifth of LDS's busy cycles; they move half as much.)
template <int kRowBytes, int kBits>
__device__ __forceinline__ int across_turn(int row)
{
    if (kBits == 8) return kRowBytes == 256 ? (row & 7) | ((row >> 1) & 8) : ((row >> 1) & 3) | ((row >> 2) & 4);
    return kRowBytes == 128 ? (row >> 1) & 7 : kRowBytes == 64 ? (row >> 2) & 3 : (row >> 3) & 1;
}

// kTerms: 1 for codes of 8 or 4 bits; 2 or 3 for a gradient, whose x are binary16 terms (kXBits 16, bq_linear_bwd.hip) and whose sums are
// float32, those of the first terms and those of the others apart.
// kAcross: the weights lie with the channels contiguous, [summed index][channel], and a stage is 64 rows of them; what a lane needs, 16
// codes of one channel, comes out of LDS by reads that transpose.  Piece j of the first operand is then channels 16 j .. 16 j + 15; of
// 2-bit codes, which are read as fields of 4 bits, the even or (odd j) the odd ones of 32 (j / 2) .. 32 (j / 2) + 31.
template <int kXBits, int kWBits, int kTerms, typename Shape, bool kAcross = false>
__global__ __launch_bounds__(Shape::threads, 2) void linear_tile_kernel(LinearArgs A)
{
    typedef TileStages<kXBits, kWBits, Shape> Stages;
    constexpr int kSteps = Stages::steps, kDepth = Stages::depth;
    constexpr int kXRow = Stages::x_row, kWRow = Stages::w_row;
    constexpr bool kFloat = kXBits == 16;
    static_assert(kFloat == (kTerms > 1) && (!kFloat || kAcross || kWBits == 8), "codes, or a gradient");
    typedef typename SumType<kFloat>::type Sum;
    constexpr int kXWords = kXRow / 16, kWWords = kWRow / 16 < 2 ? 2 : kWRow / 16;  // of a lane: a quarter of every row of 16
    constexpr int kWLine = kAcross ? Shape::w_rows * kWBits / 8 : kWRow;  // bytes of w's rows in LDS
    static_assert(!kAcross || kFloat, "a gradient");
    constexpr int kXBytes = Shape::x_rows * kXRow, kWBytes = Shape::w_rows * kWRow, kStage = kXBytes + kWBytes;
    constexpr int kXLoads = kXBytes / 1024 / Shape::waves, kWCount = kWBytes / 1024, kWLoads = (kWCount + Shape::waves - 1) / Shape::waves;
    static_assert(kXLoads * 1024 * Shape::waves == kXBytes && (kWCount % Shape::waves == 0 || Shape::waves % kWCount == 0),
                  "whole loads per wave, or some waves load the same");
    static_assert(Shape::pieces % kTerms == 0, "terms of a token in one wave");
    constexpr int kTokens = Shape::x_rows / kTerms, kP = Shape::pieces;
    constexpr bool kNatural = kXBits != kWBits;
    extern __shared__ __align__(16) uint8_t tile_lds[];

    // which tile: workgroups go round the 8 XCDs, each of which takes a contiguous eighth of the tiles; within it 8 tiles along the
    // tokens and then the next channels, so that what runs together shares its rows in the XCD's L2
    const uint32_t n_tiles = (uint32_t)(A.n + Shape::w_rows - 1) / Shape::w_rows;
    const int64_t most = row_tiles_bound(A, kTokens), counted = row_tiles(A, kTokens);  // (more only of overlapping experts)
    const uint32_t m_tiles = (uint32_t)(counted < most ? counted : most);
    const uint32_t all = m_tiles * n_tiles, each = (all + 7) / 8, idx = blockIdx.x >> 3;
    const uint32_t tile = (blockIdx.x & 7) * each + idx;
    if (idx >= each || tile >= all) return;
    const uint32_t band = tile / (8 * n_tiles), in_band = tile - band * (8 * n_tiles);
    const uint32_t band_rows = m_tiles - band * 8 < 8 ? m_tiles - band * 8 : 8;
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
        const int plane = kTerms == 1 ? 0 : (q * (1024 / kXRow) / 16) % kTerms;
        const int token = kTerms == 1 ? row : (row / (16 * kTerms)) * 16 + row % 16;
        const int last = (int)(rt.row_end - rt.row0) - 1;
        x_piece[i] = (lane % (kXRow / 16)) ^ lds_turn<kXRow, kXWords / 4>(row);
        x_base[i] = A.x + plane * A.plane_step + rt.row0 * A.ldx;
        x_off[i] = (uint32_t)(token < last ? token : last) * (uint32_t)A.ldx + x_piece[i] * 16;
    }
    const int w_wave = kWCount < Shape::waves ? wave % kWCount : wave;
    w_base = A.w + rt.expert * A.w_step + (kAcross ? (int64_t)o0 * kWBits / 8 : (int64_t)o0 * A.ldw);
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
        const int row = (i * Shape::waves + w_wave) * (1024 / kWLine) + lane / (kWLine / 16);
        if constexpr (kAcross) {
            const int piece = (lane % (kWLine / 16)) ^ across_turn<kWLine, kWBits>(row), last = (int)((int64_t)(A.n - o0) * kWBits / 128) - 1;
            w_piece[i] = row;
            w_off[i] = (uint32_t)row * (uint32_t)A.ldw + (piece < last ? piece : last) * 16;
        } else {
            const int last = A.n - o0 - 1;
            w_piece[i] = (lane % (kWRow / 16)) ^ w_turn<kWRow>(row);
            w_off[i] = (uint32_t)(row < last ? row : last) * (uint32_t)A.ldw + w_piece[i] * 16;
        }
    }
    const int stages = (A.k + Stages::codes - 1) / Stages::codes;
    const int x_tail = (int)((int64_t)A.k * kXBits / 128) % (kXRow / 16), w_tail = (int)((int64_t)A.k * kWBits / 128) % (kWRow / 16);  // pieces of the last stage
    constexpr int kLoads = kXLoads + kWLoads;
    auto load = [&](int s, int place, int n) {  // the n-th of stage s's loads, into a place of the ring
        const uint32_t at = lds0 + place * kStage + wave * 1024;
        if (n < kXLoads) {
            const bool missing = x_tail && s == stages - 1 && x_piece[n] >= x_tail;  // a piece behind the last input: any other one
            load_to_lds(at + n * Shape::waves * 1024, missing ? x_off[n] - x_piece[n] * 16 : x_off[n], x_base[n] + (int64_t)s * kXRow);
        } else if constexpr (kAcross) {
            // rows behind the last: the last one (the terms there are 0)
            const int i = n - kXLoads, behind = s == stages - 1 ? s * Stages::codes + w_piece[i] - (A.w_rows - 1) : 0;
            load_to_lds(at + kXBytes + (i * Shape::waves + w_wave - wave) * 1024, w_off[i] - (behind > 0 ? behind * (uint32_t)A.ldw : 0u),
                        w_base + (int64_t)s * Stages::codes * A.ldw);
        } else {
            const int i = n - kXLoads;
            const bool missing = w_tail && s == stages - 1 && w_piece[i] >= w_tail;
            load_to_lds(at + kXBytes + (i * Shape::waves + w_wave - wave) * 1024, missing ? w_off[i] - w_piece[i] * 16 : w_off[i], w_base + (int64_t)s * kWRow);
        }
    };

    // What a lane reads of a stage: 16 or 32 codes of every 16-row piece of x and of w, as they lie.  f of a lane's rows is the same for all
    // pieces, so the pieces are constant offsets apart.
    const int x_row = wave_t * kP * 16 + r16, w_row = wave_n * 64 + 16 * (r16 >> 2) + (r16 & 3);
    auto read_x = [&](int place, int i, int h, uint32_t (&v)[kXWords]) {  // 16 bytes
        const uint4 q = *(const uint4 *)(tile_lds + place * kStage + (x_row + i * 16) * kXRow +
                                         (((kXWords == 8 ? 2 * g : g) + h) ^ lds_turn<kXRow, kXWords / 4>(r16)) * 16);
        v[4 * h] = q.x; v[4 * h + 1] = q.y; v[4 * h + 2] = q.z; v[4 * h + 3] = q.w;
    };
    // (across: the address that a lane gives is another one's row)
    const int across_row = 16 * g + (kWBits == 8 ? r16 >> 1 : r16);
    const int across_at = across_row * kWLine + ((wave_n * (kWBits / 2)) ^ across_turn<kWLine, kWBits>(across_row)) * 16 +
                          (kWBits == 8 ? r16 & 1 : 0) * 8;
    auto read_w = [&](int place, int n, int h, uint32_t (&v)[4][kWWords]) {
        const int j = n % 4;
        if constexpr (kAcross) {
            const int half = kWBits == 8 ? 0 : j % 2 * 8, piece = kWBits == 8 ? j : kWBits == 4 ? j / 2 : 0;
            const int at = place * kStage + kXBytes + (across_at ^ (piece * 16)) + half + h * 8 * kWLine;
            typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
            i32x2 q;
            if constexpr (kWBits == 8)
                q = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(tile_lds + at));
            else
                q = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(tile_lds + at));
            v[j][2 * h] = (uint32_t)q[0]; v[j][2 * h + 1] = (uint32_t)q[1];
            return;
        }
        const uint8_t *p = tile_lds + place * kStage + kXBytes + (w_row + j * 4) * kWRow;
        if constexpr (kWBits == 2) {
            const uint2 q = *(const uint2 *)(p + ((g >> 1) ^ w_turn<kWRow>(w_row)) * 16 + (g & 1) * 8);
            v[j][0] = q.x; v[j][1] = q.y;
        } else {
            const uint4 q = *(const uint4 *)(p + (((kWWords == 8 ? 2 * g : g) + h) ^ w_turn<kWRow>(w_row)) * 16);
            v[j][4 * h] = q.x; v[j][4 * h + 1] = q.y; v[j][4 * h + 2] = q.z; v[j][4 * h + 3] = q.w;
        }
    };
    // codes behind the last input count as 0 (then the weights' do not matter)
    auto clear_tail = [&](int s, int place) {
        if (!x_tail || s != stages - 1) return;
        for (int p = threadIdx.x; p < Shape::x_rows * (kXRow / 16); p += Shape::threads) {
            const int row = p / (kXRow / 16), at = p % (kXRow / 16);
            if ((at ^ lds_turn<kXRow, kXWords / 4>(row)) >= x_tail) *(uint4 *)(tile_lds + place * kStage + row * kXRow + at * 16) = make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
    };

    // The reads run two pieces ahead of the products.  Once the last piece of a stage has been read, its place is free for the stage
    // kDepth further on; the products of the last two pieces cover the first reads of the next stage.  Reads and loads stand one
    // by one between the products (four of them each), in the order written here: a wave issues in order, and in one burst behind
    // the barrier the reads of 8 waves would hold up everyone's products.
    constexpr int kRing = kP == 2 ? 2 : kP % 4 == 0 ? 4 : 3, kX = kP == 2 ? 2 : 1;  // (two pieces are all read ahead: x alternates like w)
    static_assert(kP % kRing == 0, "the ring's places are the same in every stage");
    constexpr int kWTurns = (kAcross && kWBits == 8) || kWWords == 8 ? 2 : 1, kWEach = kAcross && kWBits == 2 ? 2 : 4;
    constexpr int kXReads = kXWords / 4, kWReads = kWTurns * kWEach;  // of a piece of x; of all of w
    constexpr int kFirst = kWReads + 2 * kXReads;  // reads that a stage starts from
    constexpr int kSums = kFloat ? kP / kTerms * 2 : kP;
    Sum acc[kSums][4] = {};
    uint32_t wv[2][4][kWWords], xv[kX][kRing][kXWords];  // (w's codes alternate: in one array every stage began by copying them)
    auto first_read = [&](int place, int n, uint32_t (&wv)[4][kWWords], uint32_t (&xv)[kRing][kXWords]) {
        // w's first halves, x's first piece, w's other halves, x's second piece
        if (n < kWEach)
            read_w(place, n, 0, wv);
        else if (n < kWEach + kXReads)
            read_x(place, 0, n - kWEach, xv[0]);
        else if (n < kWReads + kXReads)
            read_w(place, n - kWEach - kXReads, 1, wv);
        else
            read_x(place, 1, n - kWReads - kXReads, xv[1]);
    };
    // LEFT: 2 in the ring's steady state, 1 behind the last load, 0 the last
    auto stage = [&](int s, int place, int next_place, const uint32_t (&wv)[4][kWWords], uint32_t (&wn)[4][kWWords], uint32_t (&xv)[kRing][kXWords],
                     uint32_t (&xn)[kRing][kXWords], auto LEFT) {
        constexpr int left = decltype(LEFT)::value;
        i32x4 a[kSteps][4];
#pragma unroll
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (kAcross)
                    a[h][j] = kWBits == 8 ? half_codes8(wv[j][2 * h], wv[j][2 * h + 1]) : kWBits == 4 ? half_codes4(wv[j][h]) : half_codes2(wv[j / 2][h], j % 2);
                else if constexpr (kFloat)
                    a[h][j] = half_codes8(wv[j][2 * h], wv[j][2 * h + 1]);
                else
                    a[h][j] = step_codes<kWBits, kNatural>(wv[j], h);
            }
        i32x4 b = step_codes<kXBits == 16 ? 8 : kXBits, kNatural>(xv[0], 0);
#pragma unroll
        for (int q = 0; q < kSteps * kP; ++q) {
            constexpr int kOver = 2 * kSteps, kTurn = kSteps * kP - kOver;  // from here on the reads belong to the next stage
            const int i = q / kSteps, h = q % kSteps;
            if (q < kTurn) {
                if (h < kXReads) read_x(place, i + 2, h, xv[(i + 2) % kRing]);
            } else if constexpr (left > 0) {
                if (q == kTurn) {
                    // this wave's loads of stage s + 1 have landed and its reads of stage s are done; with the barrier, everyone's
                    if constexpr (left == 2)
                        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((kDepth - 2) * kLoads) : "memory");
                    else
                        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    if (left == 1) clear_tail(s + 1, next_place);
                }
                if constexpr (left == 2) {
#pragma unroll
                    for (int n = (q - kTurn) * kLoads / kOver; n < (q - kTurn + 1) * kLoads / kOver; ++n) load(s + kDepth, place, n);
                }
#pragma unroll
                for (int n = (q - kTurn) * kFirst / kOver; n < (q - kTurn + 1) * kFirst / kOver; ++n) first_read(next_place, n, wn, xn);
            }
            i32x4 next = b;
            if (q + 1 < kSteps * kP) next = step_codes<kXBits == 16 ? 8 : kXBits, kNatural>(xv[((q + 1) / kSteps) % kRing], (q + 1) % kSteps);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Sum &sum = acc[kFloat ? i / kTerms * 2 + (i % kTerms != 0) : i][j];
                sum = multiply(a[h][j], b, sum);
            }
            b = next;
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    static_assert(kDepth >= 2 && (kDepth - 1) * kLoads < 64, "the wait's counter has 6 bits");
    for (int s = 0; s < kDepth && s < stages; ++s) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) load(s, s, n);
    }
    if (stages >= kDepth)
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((kDepth - 1) * kLoads) : "memory");
    else
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    clear_tail(0, 0);
#pragma unroll
    for (int n = 0; n < kFirst; ++n) first_read(0, n, wv[0], xv[0]);
    auto after = [&](int place) { return place + 1 == kDepth ? 0 : place + 1; };
    auto even_again = [&] {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < kWWords; ++v) wv[0][j][v] = wv[1][j][v];
#pragma unroll
        for (int i = 0; i < kRing; ++i)
#pragma unroll
            for (int v = 0; v < kXWords; ++v) xv[0][i][v] = xv[kX - 1][i][v];
    };
    int s = 0, place = 0;
    for (; s + kDepth + 1 < stages; s += 2) {
        const int second = after(place), third = after(second);
        stage(s, place, second, wv[0], wv[1], xv[0], xv[kX - 1], std::integral_constant<int, 2>{});
        stage(s + 1, second, third, wv[1], wv[0], xv[kX - 1], xv[0], std::integral_constant<int, 2>{});
        place = third;
    }
    if (s + kDepth < stages) {
        stage(s, place, after(place), wv[0], wv[1], xv[0], xv[kX - 1], std::integral_constant<int, 2>{});
        even_again();
        place = after(place);
        ++s;
    }
    for (; s + 1 < stages; ++s) {
        stage(s, place, after(place), wv[0], wv[1], xv[0], xv[kX - 1], std::integral_constant<int, 1>{});
        even_again();
        place = after(place);
    }
    stage(s, place, 0, wv[0], wv[1], xv[0], xv[kX - 1], std::integral_constant<int, 0>{});

    // (all loads in flight together: one after another, a token's scale at a time, they were a third of the time behind the last stage)
    constexpr int kOut = kP / kTerms;
    const int64_t t0 = rt.row0 + wave_t * kOut * 16 + r16;
    int64_t token[kOut];
#pragma unroll
    for (int i = 0; i < kOut; ++i) token[i] = t0 + 16 * i < rt.row_end ? t0 + 16 * i : rt.row_end - 1;
    if constexpr (kFloat) {  // a gradient has no scales and no bias of the channels
        // neighbouring channels of a lane: 16, or as many as the pieces of weights that lie across leave together
        constexpr int kRun = !kAcross ? 16 : kWBits == 2 ? 8 : 4, kRuns = 16 / kRun;
        const int o = o0 + wave_n * 64 + g * kRun;
        int exponent[kOut];
#pragma unroll
        for (int i = 0; i < kOut; ++i) exponent[i] = ((const int *)A.xs)[token[i]];
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            const int64_t t = t0 + 16 * i;
            if (t >= rt.row_end) continue;
#pragma unroll
            for (int j = 0; j < kRuns; ++j) {
                const int first = o + 4 * kRun * j;
                if (first >= A.n) continue;
                float v[kRun];
#pragma unroll
                for (int r = 0; r < kRun; ++r) {
                    const int piece = kRun == 16 ? r / 4 : kRun == 8 ? 2 * j + r % 2 : j, at = kRun == 8 ? r / 2 : r % 4;
                    v[r] = ldexpf(terms_sum(acc[2 * i][piece][at], acc[2 * i + 1][piece][at]) * A.factor, exponent[i]);
                }
                store_results<kRun>(A, t * A.ldy + first, v, A.n - first);
            }
        }
    } else {
        const int o = o0 + wave_n * 64 + g * 16;
        if (o >= A.n) return;
        float xs[kOut], ws[16], bias[16];
        int64_t channel[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) channel[c] = (int64_t)rt.expert * A.n + (o + c < A.n ? o + c : A.n - 1);
        load_scales(A.xs, A.xs_f16, token, xs);
        load_scales(A.ws, A.ws_f16, channel, ws);
        channel_bias(A, channel, bias);
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            if (t0 + 16 * i >= rt.row_end) continue;
            float v[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) v[c] = scaled(acc[i][c >> 2][c & 3], A.factor, xs[i], ws[c]);
            if (A.bias) {
#pragma unroll
                for (int c = 0; c < 16; ++c) v[c] += bias[c];
            }
            store_results<16>(A, (t0 + 16 * i) * A.ldy + o, v, A.n - o);
        }
    }
}

template <int kXBits, int kWBits, int kTerms, typename Shape, bool kAcross = false>
hipError_t launch_tile(const LinearArgs &A, hipStream_t stream)
{
    constexpr size_t kLds = (size_t)TileStages<kXBits, kWBits, Shape>::depth * TileStages<kXBits, kWBits, Shape>::bytes;
    static LdsLimitOnce limit;
    const hipError_t e = limit.set((const void *)linear_tile_kernel<kXBits, kWBits, kTerms, Shape, kAcross>, kLds);
    if (e != hipSuccess) return e;
    const int64_t n_tiles = (A.n + Shape::w_rows - 1) / Shape::w_rows;
    const int64_t all = row_tiles_bound(A, Shape::x_rows / kTerms) * n_tiles;
    hipLaunchKernelGGL((linear_tile_kernel<kXBits, kWBits, kTerms, Shape, kAcross>), dim3((unsigned)((all + 7) / 8 * 8)), dim3(Shape::threads), kLds,
                       stream, A);
    return hipGetLastError();
}

}  // namespace bq
