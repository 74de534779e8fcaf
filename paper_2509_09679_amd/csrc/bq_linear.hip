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
// (11008, 4096), (8192, 8192) and (4096, 32000), codes of 8, 4 and 2 bits): what they choose is within 2 % of the best of the
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
double rows_us(const LinearArgs &A, int xbits, int wbits, int blocks, int cols)
{
    const double rounds = pieces(A, 16 * blocks) * std::ceil(A.n / (16.0 * cols)) / kCUs;
    const double kb = (16.0 * blocks * xbits + 16.0 * cols * (wbits == 8 ? 8.0 : wbits == 4 ? 4.8 : 4.4)) / 8.0 * A.k / 1000.0;
    const double codes = (rounds > 1.0 ? rounds : 1.0) * ((blocks * cols >= 8 ? 2.1 : 1.1) + kb / 50.0);
    const double weights = weights_us(A, wbits);
    return 1.55 + (codes > weights ? codes : weights);
}

// A round of tiles on all compute units: `fixed` us and `stage` us per 128 codes.
double tile_us(const LinearArgs &A, int wbits, int x_rows, int channels, double at_once, double fixed, double stage)
{
    const double tiles = pieces(A, x_rows) * std::ceil((double)A.n / channels);
    const double codes = std::ceil(tiles / at_once) * (fixed + stage * A.k / 128.0), weights = weights_us(A, wbits);
    return 2.15 + (codes > weights ? codes : weights);
}

Choice choose_codes(const LinearArgs &A, int xbits, int wbits)
{
    Choice c{1e30, true, 1, 1, kTileLarge};
    auto rows = [&](int b, int n) {
        const double us = rows_us(A, xbits, wbits, b, n);
        if (us < c.us) c = Choice{us, true, b, n, kTileLarge};
    };
    auto tiles = [&](LinearTile which, double us) {
        if (us < c.us) c = Choice{us, false, 0, 0, which};
    };
    rows(1, 1);
    rows(1, 2);
    rows(2, 1);
    rows(2, 2);
    rows(1, 4);
    rows(4, 2);
    tiles(kTileLarge, tile_us(A, wbits, 256, 256, kCUs, 5.35, 1.50));
    if (xbits == 8) tiles(kTileTall, tile_us(A, wbits, 192, 256, kCUs, 4.3, 1.33));
    tiles(kTileMiddle, tile_us(A, wbits, 128, 256, kCUs, 3.1, 0.93));
    tiles(kTileSmall, tile_us(A, wbits, 128, 128, 2.0 * kCUs, 4.2, 0.93));
    // one on a compute unit: eight waves with all of its LDS (512 tokens, 4096 -> 4096: 20.3 us, four waves 22.3 us), but packed
    // weights, which every wave along the tokens unpacks for itself, stay with four (22.1, eight waves 23.0 us)
    if (wbits == 8)
        tiles(kTileDeep, tile_us(A, wbits, 128, 128, kCUs, 3.5, 0.52));
    else
        tiles(kTileSmall, tile_us(A, wbits, 128, 128, kCUs, 4.4, 0.66));
    return c;
}

// Gradients: a fit of the same kind to a sweep of their kernels (1 .. 8192 tokens, (N, K) from (320, 11008) and (512, 1024) to (11008, 4096)
// and (8192, 8192), two and three terms, weights of 8, 4 and 2 bits as they lie and transposed).  What it chooses is within 1 % of the sweep's
// best on average; the worst is 19 % off it where that takes more than 10 us.  Measured, 8-bit weights as they lie (few rows:
// transposed) 4096 -> 4096, us:
//   two terms, tokens       8    32   128   256   512  1024  2048  4096  8192
//   1x1                   7.4    13    34    61   112
//   2x2                    11    14    21    35    62
//   64 x 128 deep          39    39    40    41    46    87   174   330   657
//   64 x 128               39    40    41    42    46    71   136   265   515
//   64 x 256               52    54    55    56    57    68   132   260   515
//   96 x 256               65    66    69    69    70    74   150   240   472
//   128 x 256              80    81    84    85    84    86   104   214   412
//   three terms, 64 x 128  47    48    49    50    60   115   225   438
//   three terms, 128 x 128 66    67    71    71    71    85   174   340
struct TermsTile {
    LinearTile tile;
    int tokens, channels;
    double at_once;
    struct {
        double launch, fixed, stage, least;  // us: of all, of a tile, of 64 outputs of a tile; of a last round that is half full or less
    } turned, across;
};
constexpr TermsTile kTwoTerms[] = {{kTileLarge, 128, 256, kCUs, {0.5, 6.7, 1.48, 0.76}, {0.9, 7.5, 1.43, 0.82}},
                                   {kTileTall, 96, 256, kCUs, {1.5, 4.9, 1.16, 0.78}, {1.6, 5.6, 1.16, 0.83}},
                                   {kTileMiddle, 64, 256, kCUs, {1.8, 3.6, 0.86, 0.81}, {1.9, 4.1, 0.89, 0.86}},
                                   {kTileSmall, 64, 128, 2.0 * kCUs, {3.1, 2.1, 0.93, 0.54}, {3.5, 2.9, 0.95, 0.58}},
                                   {kTileDeep, 64, 128, kCUs, {1.4, 3.0, 0.59, 0.90}, {1.8, 3.4, 0.60, 0.91}}};
constexpr TermsTile kThreeTerms[] = {{kTileLarge, 128, 128, kCUs, {-1.1, 8.2, 1.26, 0.75}, {1.0, 5.5, 1.26, 0.81}},
                                     {kTileDeep, 64, 128, kCUs, {1.1, 4.3, 0.77, 0.81}, {1.8, 3.3, 0.79, 0.87}}};

double terms_tile_us(const LinearArgs &A, int wbits, const TermsTile &t, bool across)
{
    const auto &c = across ? t.across : t.turned;
    const double rounds = pieces(A, t.tokens) * std::ceil((double)A.n / t.channels) / t.at_once, whole = std::floor(rounds), part = rounds - whole;
    const double last = part == 0.0 ? 0.0 : part < 0.5 ? c.least : c.least + (1.0 - c.least) * (2.0 * part - 1.0);
    const double us = (whole + last) * (c.fixed + c.stage * A.k / 64.0), weights = weights_us(A, wbits);
    return c.launch + (us > weights ? us : weights);
}

// a workgroup's us per 1000 outputs: of a row of terms, of a column of weights, of their products
double terms_rows_us(const LinearArgs &A, int terms, int blocks, int cols)
{
    const double rounds = pieces(A, 16 * blocks) * std::ceil(A.n / (16.0 * cols)) / kCUs;
    const double us = (terms == 2 ? 0.254 * blocks * 2 + 0.307 * cols + 0.068 * blocks * 2 * cols : 0.286 * blocks * 3 + 0.137 * blocks * 3 * cols) * A.k / 1000.0;
    const double all = (rounds > 1.0 ? rounds : 1.0) * (0.5 + us), weights = weights_us(A, 8);
    return 2.4 + (all > weights ? all : weights);
}

Choice choose_terms(const LinearArgs &A, int wbits, int terms, bool across)
{
    Choice c{1e30, true, 1, 1, kTileLarge};
    for (int b = 1; b <= 2 && !across; ++b)
        for (int n = 1; n <= 2; ++n) {
            if (terms == 3 && b == 2 && n == 2) continue;
            const double us = terms_rows_us(A, terms, b, n);
            if (us < c.us) c = Choice{us, true, b, n, kTileLarge};
        }
    auto tile = [&](const TermsTile &t) {
        if (across && wbits < 8 && terms == 2 && t.tile == kTileDeep) return;  // (four waves, which unpack half as much, are as quick)
        const double us = terms_tile_us(A, wbits, t, across);
        if (us < c.us) c = Choice{us, false, 0, 0, t.tile};
    };
    if (terms == 2)
        for (const TermsTile &t : kTwoTerms) tile(t);
    else
        for (const TermsTile &t : kThreeTerms) tile(t);
    return c;
}

}  // namespace

hipError_t launch_linear(const LinearArgs &A0, int xbits, int wbits, hipStream_t stream)
{
    LinearArgs A = A0;
    A.factor /= (float)((1 << (8 - xbits)) * (1 << (8 - wbits)));
    if (!fast_layout(A, xbits, wbits)) return launch_linear_any(A, xbits, wbits, stream);
    const Choice c = choose_codes(A, xbits, wbits);
    if (c.few) {
        if (xbits == 4) return launch_linear_rows4(A, wbits, c.blocks, c.cols, stream);
        return launch_linear_rows8(A, wbits, c.blocks, c.cols, stream);
    }
    if (xbits == 8) return launch_linear_tile8(A, wbits, c.tile, stream);
    return launch_linear_tile4(A, wbits, c.tile, stream);
}

hipError_t launch_linear_terms(const LinearArgs &A, int terms, hipStream_t stream)
{
    const Choice c = choose_terms(A, 8, terms, false);
    return c.few ? launch_linear_rows_terms(A, terms, c.blocks, c.cols, stream) : launch_linear_tile_terms(A, terms, c.tile, stream);
}

// Weights as they lie save the transposition, its bytes at what the launch reaches that writes terms and transposes.
bool linear_across_is_quicker(const LinearArgs &across, const LinearArgs &turned, int wbits, int terms)
{
    if ((uintptr_t)across.w % 16 != 0 || across.ldw % 16 != 0 || across.n * (int64_t)wbits % 128 != 0 || across.ldw >= (int64_t)1 << 23) return false;
    const double used = !across.offsets ? 1.0 : across.experts < across.rows ? across.experts : (double)across.rows;
    const double transposition = used * across.n * (across.k + across.w_rows * wbits / 8.0) / 5.0e6;
    return choose_terms(across, wbits, terms, true).us < choose_terms(turned, 8, terms, false).us + transposition;
}

hipError_t launch_linear_across(const LinearArgs &A, int wbits, int terms, hipStream_t stream)
{
    return launch_linear_tile_across(A, wbits, terms, choose_terms(A, wbits, terms, true).tile, stream);
}

}  // namespace bq
