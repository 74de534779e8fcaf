// Which kernel takes a product of codes or a gradient, and the shapes there are: rules on sizes alone, for the host (no HIP in here).
#pragma once

#include <cmath>
#include <cstdint>

namespace bq {

struct LinearSize {
    int64_t rows;
    int k, n, experts;  // summed index and channels
    bool grouped;
    int w_rows;         // of a gradient's weights: the summed index without padding
};

enum LinearTile { kTileLarge, kTileTall, kTileMiddle, kTileSmall, kTileDeep };

struct LinearChoice {
    double us;
    bool few;
    int blocks, cols;  // of the kernel for few rows
    LinearTile tile;
};

// ---- shapes: few rows (bq_linear_rows.h) ----------------------------------------------------------------------

// kWide: all of a compute unit's LDS for one workgroup, else half of it.
template <int kXBits, int kWBits, int kTerms, int kBlocks, int kCols, bool kWide>
struct RowsShape {
    static constexpr int frags = kBlocks * kTerms;
    static constexpr int codes = kXBits == 16 ? 64 : kWBits == 2 ? 256 : 128;   // of a step
    static constexpr int x_row = codes * kXBits / 8, w_row = codes * kWBits / 8;  // bytes of a step's rows: 64, 128, 256
    static constexpr int x_bytes = frags * 16 * x_row, w_bytes = kCols * 16 * w_row, step = x_bytes + w_bytes;
    static constexpr int room = (kWide ? 160 : 80) * 1024;
    static constexpr int waves = 16 * step <= room ? 8 : 4;
    static constexpr int per_simd = kWide ? 2 : waves / 2;  // waves that have to fit (four alone would get registers they have no use for)
    static constexpr int fit = room / (waves * step), depth = fit < 4 ? fit : 4;
    static constexpr int pairs = kBlocks * kCols, chunk = pairs < waves ? pairs : waves;  // pieces joined at a time
    static constexpr int joined = waves * chunk * 1024;
    static constexpr int lds = waves * depth * step > joined ? waves * depth * step : joined;
    static constexpr bool exists = depth >= 2;  // one step is multiplied while another is loaded
};

struct RowsGrid {
    int64_t along_channels, along_rows, experts;
};

inline RowsGrid rows_grid(const LinearSize &A, int blocks, int cols)
{
    // by expert: as many workgroups along the rows as an expert needs that has twice its share; they go on where it has more
    const int64_t rows = A.grouped ? (2 * A.rows + A.experts - 1) / A.experts : A.rows;
    const int64_t passes = (rows + 16 * blocks - 1) / (16 * blocks);
    return RowsGrid{(A.n + 16 * cols - 1) / (16 * cols), passes < 1024 ? passes : 1024, A.experts};
}

// Two workgroups on a compute unit hide one another's first loads and last sums; one alone gets more loads in flight.  8-bit codes
// of 16 tokens, K = 4096: 256 workgroups 7.4 us in pairs and 6.6 us alone, 688 of them 14.5 and 16.6 us.  Packed weights leave
// room for deep rings either way (688 workgroups 9.9 and 12.6 us, 256 of them 4.6 and 4.8 us) and never have one alone.
inline bool rows_alone(const RowsGrid &g) { return g.along_channels * g.along_rows * g.experts <= 256; }

// ---- shapes: tiles (bq_linear_tile.h) -------------------------------------------------------------------------

// Waves of a workgroup along tokens and channels, 16-row pieces of a wave along tokens (of x's rows: terms count); 64 channels per wave.
// kLds: what the ring may take of a compute unit's LDS, in KB.
template <int kWavesT, int kWavesN, int kPieces, int kLds>
struct TileShape {
    static constexpr int lds = kLds * 1024;
    static constexpr int waves_t = kWavesT, waves_n = kWavesN, pieces = kPieces;
    static constexpr int waves = kWavesT * kWavesN, threads = 64 * waves;
    static constexpr int x_rows = kWavesT * kPieces * 16, w_rows = kWavesN * 64;
};

constexpr int kMostStages = 4;

// The ring: matrix instructions along a stage's codes (64 each, of a gradient's terms 32), bytes of a stage's rows, stages that fit.
template <int kXBits, int kWBits, typename Shape>
struct TileStages {
    static constexpr int steps = 2, codes = steps * (kXBits == 16 ? 32 : 64);
    static constexpr int x_row = codes * kXBits / 8, w_row = codes * kWBits / 8;
    static constexpr int bytes = Shape::x_rows * x_row + Shape::w_rows * w_row;
    static constexpr int fit = Shape::lds / bytes;
    static constexpr int depth = fit < kMostStages ? fit : kMostStages;
};

// x rows (tokens times terms) x channels
typedef TileShape<2, 4, 8, 160> TileLarge;   // 256 x 256
typedef TileShape<2, 4, 6, 160> TileTall;    // 192 x 256, for 8-bit codes
typedef TileShape<2, 4, 4, 160> TileMiddle;  // 128 x 256
typedef TileShape<2, 2, 4, 80> TileSmall;    // 128 x 128, two workgroups per compute unit
typedef TileShape<4, 2, 2, 160> TileDeep;    // 128 x 128, one of them with eight waves and all of the LDS
typedef TileShape<4, 2, 6, 160> TileLarge3;  // 384 x 128, for three terms
typedef TileShape<4, 2, 3, 160> TileDeep3;   // 192 x 128


// ---- the choice -----------------------------------------------------------------------------------------------

constexpr double kCUs = 256.0;

// Pieces of `rows` rows that the batch makes: every expert's last one is half full on average, and none is empty.
inline double pieces(const LinearSize &A, int rows)
{
    if (!A.grouped) return std::ceil((double)A.rows / rows);
    const double used = A.experts < A.rows ? A.experts : (double)A.rows;
    const double some = (double)A.rows / rows + 0.5 * used;
    return std::ceil(some > used ? some : used);
}

// What a kernel takes, in us.  The constants below are fits to a sweep of all kernels (1 .. 8192 tokens, (K, N) from (1024, 2048) to
// (11008, 4096), (8192, 8192) and (4096, 32000), codes of 8, 4 and 2 bits).  In another sweep, of (512, 1024), (320, 11008) and batches of 8 and
// 32 experts too, what they choose takes 2 to 5 % more than the best on average where that takes more than 10 us, and at worst 20 to
// 43 %.  Measured, 8-bit codes 4096 -> 4096, us:
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
inline double weights_us(const LinearSize &A, int wbits)
{
    const double used = !A.grouped ? 1.0 : A.experts < A.rows ? A.experts : (double)A.rows;
    return used * A.n * A.k * wbits / 8.0 / 4.4e6;
}

// A compute unit reads 50 KB of codes a us, and every workgroup has a prologue and the joining of its sums.  Unpacking a weight, which every
// workgroup does for itself, counts as another 0.8 (4 bits) or 2.4 bits of it (2 bits: without that 16 x 64 looked 20 % too good).
inline double rows_us(const LinearSize &A, int xbits, int wbits, int blocks, int cols)
{
    const double rounds = pieces(A, 16 * blocks) * std::ceil(A.n / (16.0 * cols)) / kCUs;
    const double kb = (16.0 * blocks * xbits + 16.0 * cols * (wbits == 8 ? 8.0 : wbits == 4 ? 4.8 : 4.4)) / 8.0 * A.k / 1000.0;
    const double codes = (rounds > 1.0 ? rounds : 1.0) * ((blocks * cols >= 8 ? 2.1 : 1.1) + kb / 50.0);
    const double weights = weights_us(A, wbits);
    return 1.55 + (codes > weights ? codes : weights);
}

// A round of tiles on all compute units: `fixed` us and `stage` us per 128 codes.
inline double tile_us(const LinearSize &A, int wbits, int x_rows, int channels, double at_once, double fixed, double stage)
{
    const double tiles = pieces(A, x_rows) * std::ceil((double)A.n / channels);
    const double codes = std::ceil(tiles / at_once) * (fixed + stage * A.k / 128.0), weights = weights_us(A, wbits);
    return 2.15 + (codes > weights ? codes : weights);
}

inline LinearChoice choose_codes(const LinearSize &A, int xbits, int wbits)
{
    LinearChoice c{1e30, true, 1, 1, kTileLarge};
    auto rows = [&](int b, int n) {
        const double us = rows_us(A, xbits, wbits, b, n);
        if (us < c.us) c = LinearChoice{us, true, b, n, kTileLarge};
    };
    auto tiles = [&](LinearTile which, double us) {
        if (us < c.us) c = LinearChoice{us, false, 0, 0, which};
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
// and (8192, 8192), two and three terms, weights of 8, 4 and 2 bits as they lie and transposed): what it chooses takes 0.2 to 2.3 % more than the
// sweep's best on average where that takes more than 10 us, and at worst 17 %.  Measured, 8-bit weights as they lie (few rows: transposed) 4096 ->
// 4096, us:
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

inline double terms_tile_us(const LinearSize &A, int wbits, const TermsTile &t, bool across)
{
    const auto &c = across ? t.across : t.turned;
    const double rounds = pieces(A, t.tokens) * std::ceil((double)A.n / t.channels) / t.at_once, whole = std::floor(rounds), part = rounds - whole;
    const double last = part == 0.0 ? 0.0 : part < 0.5 ? c.least : c.least + (1.0 - c.least) * (2.0 * part - 1.0);
    const double stage = across && wbits < 8 ? 0.92 * c.stage : c.stage;  // (fields of packed codes take fewer instructions)
    const double us = (whole + last) * (c.fixed + stage * A.k / 64.0), weights = weights_us(A, wbits);
    return c.launch + (us > weights ? us : weights);
}

// a workgroup's us per 1000 outputs: of a row of terms, of a column of weights, of their products
inline double terms_rows_us(const LinearSize &A, int terms, int blocks, int cols)
{
    const double rounds = pieces(A, 16 * blocks) * std::ceil(A.n / (16.0 * cols)) / kCUs;
    const double us = (terms == 2 ? 0.254 * blocks * 2 + 0.307 * cols + 0.068 * blocks * 2 * cols : 0.286 * blocks * 3 + 0.137 * blocks * 3 * cols) * A.k / 1000.0;
    const double all = (rounds > 1.0 ? rounds : 1.0) * (0.5 + us), weights = weights_us(A, 8);
    return 2.4 + (all > weights ? all : weights);
}

inline LinearChoice choose_terms(const LinearSize &A, int wbits, int terms, bool across)
{
    LinearChoice c{1e30, true, 1, 1, kTileLarge};
    for (int b = 1; b <= 2 && !across; ++b)
        for (int n = 1; n <= 2; ++n) {
            if (terms == 3 && b == 2 && n == 2) continue;
            const double us = terms_rows_us(A, terms, b, n);
            if (us < c.us) c = LinearChoice{us, true, b, n, kTileLarge};
        }
    auto tile = [&](const TermsTile &t) {
        if (across && wbits < 8 && terms == 2 && t.tile == kTileDeep) return;  // (four waves, which unpack half as much, are as quick)
        const double us = terms_tile_us(A, wbits, t, across);
        if (us < c.us) c = LinearChoice{us, false, 0, 0, t.tile};
    };
    if (terms == 2)
        for (const TermsTile &t : kTwoTerms) tile(t);
    else
        for (const TermsTile &t : kThreeTerms) tile(t);
    return c;
}

// Weights as they lie save the transposition, its bytes at what the launch reaches that writes terms and transposes.  (Both with the same summed
// index and channels; of few experts' rows, those that have any.)
inline bool across_is_quicker(const LinearSize &A, int wbits, int terms)
{
    const double used = !A.grouped ? 1.0 : A.experts < A.rows ? A.experts : (double)A.rows;
    const double transposition = used * A.n * (A.k + A.w_rows * wbits / 8.0) / 5.0e6;
    return choose_terms(A, wbits, terms, true).us < choose_terms(A, 8, terms, false).us + transposition;
}

}  // namespace bq
