// Which kernel a product or a gradient takes, and its ring, for the tests: the library's own rules (bq_linear_choice.h), compiled for the host.
#include "bq_linear_choice.h"

using namespace bq;

namespace {

struct Ring {
    int waves, depth, codes;  // waves that share the sum (1: tiles), places of a ring, codes of a stage or step
};

template <int kX, int kW, int kTerms, int kBlocks, int kCols>
Ring rows_of(const LinearSize &A, int *alone)
{
    constexpr bool kPair = RowsShape<kX, kW, kTerms, kBlocks, kCols, false>::exists;
    *alone = !kPair || (kW == 8 && rows_alone(rows_grid(A, kBlocks, kCols)));
    typedef RowsShape<kX, kW, kTerms, kBlocks, kCols, true> Wide;
    typedef RowsShape<kX, kW, kTerms, kBlocks, kCols, false> Narrow;
    return *alone ? Ring{Wide::waves, Wide::depth, Wide::codes} : Ring{Narrow::waves, Narrow::depth, Narrow::codes};
}

template <int kX, int kW, int kTerms>
Ring rows(const LinearSize &A, const LinearChoice &c, int *alone)
{
    const int shape = c.blocks * 10 + c.cols;
    if (kTerms == 1 && shape == 14) return rows_of<kX, kW, 1, 1, 4>(A, alone);
    if (kTerms == 1 && shape == 42) return rows_of<kX, kW, 1, 4, 2>(A, alone);
    if (shape == 22) return rows_of<kX, kW, kTerms, 2, 2>(A, alone);
    if (shape == 21) return rows_of<kX, kW, kTerms, 2, 1>(A, alone);
    if (shape == 12) return rows_of<kX, kW, kTerms, 1, 2>(A, alone);
    return rows_of<kX, kW, kTerms, 1, 1>(A, alone);
}

template <int kX, int kW, typename Shape>
Ring tile_of()
{
    typedef TileStages<kX, kW, Shape> S;
    return Ring{1, S::depth, S::codes};
}

template <int kX, int kW, int kTerms>
Ring tile(LinearTile t)
{
    if (kTerms == 3) return t == kTileLarge ? tile_of<kX, kW, TileLarge3>() : tile_of<kX, kW, TileDeep3>();
    if (t == kTileLarge) return tile_of<kX, kW, TileLarge>();
    if (t == kTileTall) return tile_of<kX, kW, TileTall>();
    if (t == kTileMiddle) return tile_of<kX, kW, TileMiddle>();
    if (t == kTileDeep) return tile_of<kX, kW, TileDeep>();
    return tile_of<kX, kW, TileSmall>();
}

template <int kX, int kW, int kTerms>
void describe(const LinearSize &A, const LinearChoice &c, int across, int *out)
{
    int alone = 0;
    const Ring r = c.few ? rows<kX, kW, kTerms>(A, c, &alone) : tile<kX, kW, kTerms>(c.tile);
    const int v[9] = {c.few, c.blocks, c.cols, alone, c.few ? -1 : c.tile, across, r.waves, r.depth, r.codes};
    for (int i = 0; i < 9; ++i) out[i] = v[i];
}

}  // namespace

// out: few, blocks, cols, alone on a compute unit, tile, weights as they lie, waves, depth, codes
extern "C" void linear_forward_choice(int64_t rows, int inputs, int outputs, int experts, int xbits, int wbits, int *out)
{
    const LinearSize A{rows, inputs, outputs, experts ? experts : 1, experts != 0, 0};
    const LinearChoice c = choose_codes(A, xbits, wbits);
    if (xbits == 8) {
        if (wbits == 8) describe<8, 8, 1>(A, c, 0, out);
        if (wbits == 4) describe<8, 4, 1>(A, c, 0, out);
        if (wbits == 2) describe<8, 2, 1>(A, c, 0, out);
    } else {
        if (wbits == 8) describe<4, 8, 1>(A, c, 0, out);
        if (wbits == 4) describe<4, 4, 1>(A, c, 0, out);
        if (wbits == 2) describe<4, 2, 1>(A, c, 0, out);
    }
}

// aligned: the weights' rows are whole 16-byte pieces that start at multiples of 16
extern "C" void linear_gradient_choice(int64_t rows, int outputs, int inputs, int experts, int wbits, int terms, int aligned, int *out)
{
    const LinearSize A{rows, (outputs + 63) / 64 * 64, inputs, experts ? experts : 1, experts != 0, outputs};
    const bool across = aligned && (int64_t)inputs * wbits % 128 == 0 && across_is_quicker(A, wbits, terms);
    const LinearChoice c = choose_terms(A, across ? wbits : 8, terms, across);
    if (terms == 2) {
        if (!across || wbits == 8) describe<16, 8, 2>(A, c, across, out);
        else if (wbits == 4) describe<16, 4, 2>(A, c, across, out);
        else describe<16, 2, 2>(A, c, across, out);
    } else {
        if (!across || wbits == 8) describe<16, 8, 3>(A, c, across, out);
        else if (wbits == 4) describe<16, 4, 3>(A, c, across, out);
        else describe<16, 2, 3>(A, c, across, out);
    }
}
