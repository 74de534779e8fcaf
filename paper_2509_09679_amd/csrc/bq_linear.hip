// Which kernel takes a product of codes.
#include <cmath>

#include "bq_linear.h"

namespace bq {

namespace {

constexpr double kCUs = 256.0;

bool fast_layout(const LinearArgs &A, int xbits, int wbits)
{
    // whole 16-byte pieces of both operands; offsets within a tile of 256 rows in 32 bits
    return (uintptr_t)A.x % 16 == 0 && (uintptr_t)A.w % 16 == 0 && A.ldx % 16 == 0 && A.ldw % 16 == 0 && A.k * (int64_t)xbits % 128 == 0 &&
           A.k * (int64_t)wbits % 128 == 0 && A.ldx < (int64_t)1 << 23 && A.ldw < (int64_t)1 << 23;
}

// Pieces of `rows` rows that the batch makes: every expert's last one is half full on average, and none is empty.
double pieces(const LinearArgs &A, int rows)
{
    if (!A.offsets) return std::ceil((double)A.rows / rows);
    const double used = A.experts < A.rows ? A.experts : (double)A.rows;
    const double some = (double)A.rows / rows + 0.5 * used;
    return std::ceil(some > used ? some : used);
}

// What a kernel takes, in us.  The models below are fits to a sweep (T = 1 .. 8192 tokens, (K, N) = (4096, 4096), (4096, 11008),
// (11008, 4096), (2048, 1024), (8192, 8192), codes of 8 and 4 bits); they follow it within a fifth, and what they choose is within a
// tenth of the best of the sweep's kernels.  Measured, 8-bit codes 4096 -> 4096:
//   tokens           16     64    128    256    512   1024   2048   4096   8192
//   best few-row    7.6   11.0   15.8   19.9   37.7   70.0    144    287    601
//   128 x 128       28      27     28     27     28     26     38     73    154
//   ... deep        20      20     22     21     23     24     48     98    207
//   128 x 256       26      27     29     28     29     28     37     73    147
//   256 x 256       40      43     47     50     51     48     55     64    138

// A workgroup reads its codes at 30 KB/us, all of them together at 7.5 GB/ms.
double rows_us(const LinearArgs &A, int xbits, int wbits, int planes, int blocks, int cols)
{
    const double workgroups = pieces(A, 16 * blocks) * std::ceil(A.n / (16.0 * cols));
    const double kb = (16.0 * blocks * planes * xbits + 16.0 * cols * wbits) / 8.0 * A.k / 1000.0;
    const double alone = kb / 30.0, together = workgroups * kb / 7500.0;
    return 3.0 + (alone > together ? alone : together);
}

// A round of tiles on all compute units: `fixed` us and `stage` us per 128 codes.
double tile_us(const LinearArgs &A, int planes, int x_rows, int channels, double at_once, double fixed, double stage)
{
    const double tiles = pieces(A, x_rows / planes) * std::ceil((double)A.n / channels);
    return 3.0 + std::ceil(tiles / at_once) * (fixed + stage * A.k / 128.0);
}

}  // namespace

hipError_t launch_linear(const LinearArgs &A0, int xbits, int wbits, int planes, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor /= (float)((1 << (8 - xbits)) * (1 << (8 - wbits)));
    const size_t size = A.dtype == BQ_F32 ? 4 : 2;
    A.y_quads = (uintptr_t)A.y % 16 == 0 && A.ldy * size % 16 == 0;
    if (!fast_layout(A, xbits, wbits)) return launch_linear_any(A, xbits, wbits, planes, stream);

    int blocks = 1, cols = 1;
    LinearTile tile = kTileLarge;
    bool few = true;
    double best = rows_us(A, xbits, wbits, planes, 1, 1);
    auto rows = [&](int b, int c) {
        const double us = rows_us(A, xbits, wbits, planes, b, c);
        if (us < best) {
            best = us;
            blocks = b;
            cols = c;
        }
    };
    auto tiles = [&](LinearTile which, double us) {
        if (us < best) {
            best = us;
            few = false;
            tile = which;
        }
    };
    if (wbits < 8) rows(1, 2);
    rows(2, 1);
    if (planes < 3) rows(2, 2);
    if (planes == 1) {
        rows(4, 2);
        rows(4, 4);
    } else if (planes == 2) {
        rows(2, 4);
    } else {
        rows(1, 4);
    }
    if (planes < 3) {
        tiles(kTileLarge, tile_us(A, planes, 256, 256, kCUs, 6.0, 1.65));
        tiles(kTileMiddle, tile_us(A, planes, 128, 256, kCUs, 4.0, 0.93));
        const bool packed = xbits < 8 || wbits < 8;
        // two workgroups on a compute unit, or one: packed codes have the same stages either way
        tiles(kTileSmall, tile_us(A, planes, 128, 128, 2.0 * kCUs, 4.0, 1.08));
        tiles(packed ? kTileSmall : kTileDeep, tile_us(A, planes, 128, 128, kCUs, 4.0, 0.52));
    } else {
        tiles(kTileLarge, tile_us(A, 3, 384, 128, kCUs, 5.0, 1.35));
        tiles(kTileDeep, tile_us(A, 3, 192, 128, kCUs, 4.0, 0.75));
    }
    if (few) {
        if (xbits == 4) return launch_linear_rows4(A, wbits, blocks, cols, stream);
        return launch_linear_rows8(A, wbits, planes, blocks, cols, stream);
    }
    if (planes > 1) return launch_linear_tile_digits(A, planes, tile, stream);
    if (xbits == 8) return launch_linear_tile8(A, wbits, tile, stream);
    return launch_linear_tile4(A, wbits, tile, stream);
}

}  // namespace bq
