// Which kernel takes a product of codes.
#include <cmath>

#include "bq_linear.h"

namespace bq {

namespace {

constexpr double kCUs = 256.0;

struct Choice {
    double us;
    bool few;
    int blocks, cols;
    LinearTile tile;
};

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

// What a kernel takes, in us.  The constants below are fits to a sweep of all kernels (1 .. 8192 tokens, (K, N) from (1024, 2048) to
// (11008, 4096), (8192, 8192) and (4096, 32000), codes of 8, 4 and 2 bits, digits): what they choose is within 2 % of the best of the
// sweep's kernels on average.  Measured, 8-bit codes 4096 -> 4096, us:
//   tokens          1    16    32    64   128   256   512  1024  2048  4096  8192
//   1x1           5.9   6.5   8.5  12.6  20.5  35.7  67.9   115
//   2x2           6.4   6.9   7.4   7.4  10.9  18.0  30.9  53.9
//   4x2           7.8   8.1   8.6   9.5   9.7  17.3  31.7  57.9
//   128 x 128 deep 16    16    17    18    19    20    20    22    42    85   187
//   128 x 128      23    25    26    26    27    27    28    26    36    71   152
//   128 x 256      22    23    24    26    28    28    29    27    35    71   145
//   192 x 256      32    34    35    36    38    38    40    38    40    83   138
//   256 x 256      38    40    40    41    44    47    48    45    50    62   122

// The weights' bytes, at what a kernel that has to wait for them reaches.
double weights_us(const LinearArgs &A, int wbits)
{
    const double used = !A.offsets ? 1.0 : A.experts < A.rows ? A.experts : (double)A.rows;
    return used * A.n * A.k * wbits / 8.0 / 4.4e6;
}

// A compute unit reads 50 KB of codes a us, and every workgroup has a prologue and the joining of its sums.  Unpacking a weight, which every
// workgroup does for itself, counts as another 0.8 (4 bits) or 2.4 bits of it (2 bits: without that 16 x 64 looked 20 % too good).
double rows_us(const LinearArgs &A, int xbits, int wbits, int planes, int blocks, int cols)
{
    const double rounds = pieces(A, 16 * blocks) * std::ceil(A.n / (16.0 * cols)) / kCUs;
    const double kb = (16.0 * blocks * planes * xbits + 16.0 * cols * (wbits == 8 ? 8.0 : wbits == 4 ? 4.8 : 4.4)) / 8.0 * A.k / 1000.0;
    const double codes = (rounds > 1.0 ? rounds : 1.0) * ((blocks * planes * cols >= 8 ? 2.1 : 1.1) + kb / 50.0);
    const double weights = weights_us(A, wbits);
    return 1.55 + (codes > weights ? codes : weights);
}

// A round of tiles on all compute units: `fixed` us and `stage` us per 128 codes.
double tile_us(const LinearArgs &A, int wbits, int planes, int x_rows, int channels, double at_once, double fixed, double stage)
{
    const double tiles = pieces(A, x_rows / planes) * std::ceil((double)A.n / channels);
    const double codes = std::ceil(tiles / at_once) * (fixed + stage * A.k / 128.0), weights = weights_us(A, wbits);
    return 2.15 + (codes > weights ? codes : weights);
}

Choice choose(const LinearArgs &A, int xbits, int wbits, int planes, bool across)
{
    Choice c{1e30, true, 1, 1, kTileLarge};
    auto rows = [&](int b, int n) {
        const double us = rows_us(A, xbits, wbits, planes, b, n);
        if (us < c.us) c = Choice{us, true, b, n, kTileLarge};
    };
    auto tiles = [&](LinearTile which, double us) {
        if (us < c.us) c = Choice{us, false, 0, 0, which};
    };
    if (!across) {
        rows(1, 1);
        rows(1, 2);
        rows(2, 1);
        if (planes < 3) rows(2, 2);
        if (planes == 1) {
            rows(1, 4);
            rows(4, 2);
        }
    }
    if (planes < 3) {
        tiles(kTileLarge, tile_us(A, wbits, planes, 256, 256, kCUs, 5.35, 1.50));
        if (xbits == 8) tiles(kTileTall, tile_us(A, wbits, planes, 192, 256, kCUs, 4.3, 1.33));
        tiles(kTileMiddle, tile_us(A, wbits, planes, 128, 256, kCUs, 3.1, 0.93));
        tiles(kTileSmall, tile_us(A, wbits, planes, 128, 128, 2.0 * kCUs, 4.2, 0.93));
        // one on a compute unit: eight waves with all of its LDS (512 tokens, 4096 -> 4096: 20.3 us, four waves 22.3 us), but packed
        // weights, which every wave along the tokens unpacks for itself, stay with four (22.1, eight waves 23.0 us)
        if (wbits == 8)
            tiles(kTileDeep, tile_us(A, wbits, planes, 128, 128, kCUs, 3.5, 0.52));
        else
            tiles(kTileSmall, tile_us(A, wbits, planes, 128, 128, kCUs, 4.4, 0.66));
    } else {
        tiles(kTileLarge, tile_us(A, wbits, 3, 384, 128, kCUs, 4.7, 1.24));
        tiles(kTileDeep, tile_us(A, wbits, 3, 192, 128, kCUs, 5.0, 0.62));
    }
    return c;
}

}  // namespace

hipError_t launch_linear(const LinearArgs &A0, int xbits, int wbits, int planes, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor /= (float)((1 << (8 - xbits)) * (1 << (8 - wbits)));
    if (!fast_layout(A, xbits, wbits)) return launch_linear_any(A, xbits, wbits, stream);
    const Choice c = choose(A, xbits, wbits, planes, false);
    if (c.few) {
        if (xbits == 4) return launch_linear_rows4(A, wbits, c.blocks, c.cols, stream);
        return launch_linear_rows8(A, wbits, planes, c.blocks, c.cols, stream);
    }
    if (planes > 1) return launch_linear_tile_digits(A, planes, c.tile, stream);
    if (xbits == 8) return launch_linear_tile8(A, wbits, c.tile, stream);
    return launch_linear_tile4(A, wbits, c.tile, stream);
}

// Weights across save the transposition, its bytes at what the launch reaches that writes digits and transposes; the product's reads, 8
// bytes instead of 16, make it 2 .. 4 % slower.  2048 rows of 4096 -> 4096, bf16: 8.2 + 59.2 us, transposed 13.5 + 57.7 us.
bool linear_across_is_quicker(const LinearArgs &across, const LinearArgs &turned, int wbits, int planes)
{
    if ((uintptr_t)across.w % 16 != 0 || across.ldw % 16 != 0 || across.n * (int64_t)wbits % 128 != 0 || across.ldw >= (int64_t)1 << 23) return false;
    const double used = !across.offsets ? 1.0 : across.experts < across.rows ? across.experts : (double)across.rows;
    const double transposition = used * across.n * (across.k + across.w_rows * wbits / 8.0) / 5.0e6;
    return 1.03 * choose(across, 8, wbits, planes, true).us < choose(turned, 8, 8, planes, false).us + transposition;
}

hipError_t launch_linear_across(const LinearArgs &A0, int wbits, int planes, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor /= (float)(1 << (8 - wbits));
    return launch_linear_tile_across(A, wbits, planes, choose(A, 8, wbits, planes, true).tile, stream);
}

}  // namespace bq
