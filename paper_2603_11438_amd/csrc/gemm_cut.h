// Which tile a product on the matrix units takes, and how many runs its k is split
// into: by one table of measured costs, on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace ar {
namespace dev {

constexpr int kStepK = 64;  // steps that k is counted in

// Tiles, by planes: rows and columns, and what they cost.  `busy`: us of a
// compute unit for k = 64 of a tile while it has several to work on; `alone`:
// us for the same when one tile has the unit to itself (its loads' way to the
// L2 and back is then in the open); `fit`: tiles that share a unit; `ends`: us
// before and after the products.  Measured on products of 1024 x 1024 x 4096
// (alone) and 8192 x 8192 x 8192 (busy).  The last one has three buffers, for a
// tile alone on its unit: 768 x 1024 x 5376 in four runs 19.2 us, with two
// buffers 23.7 and in 64 x 64 tiles 31.1; with two tiles to a unit it is slower
// (5376 x 1024 x 768: 23.0 us, with two buffers 18.2).
struct TileCost {
    int side;
    double busy, alone, ends;
    int fit;
};
constexpr int kTileSizes = 5;
constexpr TileCost kTiles[2][kTileSizes] = {
    {{64, 0.19, 0.32, 2.5, 2}, {128, 0.5, 0.68, 5.0, 2}, {192, 1.1, 1.1, 12.0, 1}, {256, 1.67, 1.67, 20.0, 1}, {128, 0.5, 0.5, 5.0, 1}},
    {{64, 0.4, 0.45, 3.0, 1}, {128, 1.2, 1.3, 8.0, 1}, {192, 2.8, 2.8, 14.0, 1}, {256, 4.6, 4.6, 24.0, 1}},
};

// us of a product of k = 64 * steps in tiles of kTiles[planes - 1][tile], k in
// `splits` runs.  LOWER: tiles on and below the diagonal alone.  A split product's
// runs write their sums, and a kernel of its own reads and adds them, each at about
// 6 TB/s and with 4 us to begin with.  300 x 300 x 8192, bf16: 37.3 us in one piece,
// 7.6 + 5.6 in eight; 1024 x 1024 x 4096, two planes, of the tiles on and below the
// diagonal: 32.2, and 19.8 + 8.0 in seven (of 128 x 128).
inline size_t tiles_of(int planes, int tile, size_t m, size_t n, size_t batch, bool lower)
{
    const size_t side = (size_t)kTiles[planes - 1][tile].side, a = (m + side - 1) / side, b = (n + side - 1) / side;
    return batch * (lower ? a * (a + 1) / 2 : a * b);
}
inline double product_us(int planes, int tile, size_t m, size_t n, size_t steps, size_t batch, bool lower, uint32_t splits)
{
    const TileCost &c = kTiles[planes - 1][tile];
    const size_t tiles = tiles_of(planes, tile, m, n, batch, lower), units = (tiles * splits + 255) / 256;
    const double busy = units * c.busy, alone = (double)((units + c.fit - 1) / c.fit) * c.alone;
    double sum = ((steps + splits - 1) / splits) * (busy > alone ? busy : alone) + c.ends * units;
    if (splits > 1) sum += 4.0 + 2.0 * splits * tiles * c.side * c.side * 4 / 6e6;
    return sum;
}
// Whether k may be split so: two steps at least to a run, and some 1000 runs at most.
inline bool may_split(size_t tiles, size_t steps, uint32_t splits)
{
    return splits == 1 || (splits * 2 <= (steps > 2 ? steps : 2) && tiles * splits <= 1024);
}

// The tile and the number of runs that finish a product first, of the tiles `least`
// .. `most`.
struct Cut {
    int tile;
    uint32_t splits;
};
inline Cut cut_for(int planes, size_t m, size_t n, size_t steps, size_t batch, bool lower, int least, int most, uint32_t max_splits)
{
    Cut best{least, 1};
    double time = product_us(planes, least, m, n, steps, batch, lower, 1);
    for (int t = least; t <= most; ++t) {
        const size_t tiles = tiles_of(planes, t, m, n, batch, lower);
        for (uint32_t s = 1; s <= max_splits && may_split(tiles, steps, s); ++s) {
            const double us = product_us(planes, t, m, n, steps, batch, lower, s);
            if (us < time) best = {t, s}, time = us;
        }
    }
    return best;
}

// ---- whose tiles ------------------------------------------------------------

constexpr uint32_t kMaxSplits = 32;

// The gated feed-forward block's backward products, with `hidden` rounded up to
// kStepK.  dx: tokens x dim over dG and dU; the weights' gradients as one.
inline Cut dx_cut(size_t tokens, size_t dim, size_t hidden)
{
    return cut_for(1, tokens, dim, 2 * (hidden / kStepK), 1, false, 0, 4, kMaxSplits);
}
inline Cut dw_cut(size_t tokens, size_t dim, size_t hidden)
{
    return cut_for(1, 2 * hidden, dim, (tokens + kStepK - 1) / kStepK, 1, false, 0, 4, kMaxSplits);
}

// The products of an orthogonalising step, m <= n, with mp and np m and n rounded up
// to kStepK: A = X X^T over n, B = A A and B X over m.
inline Cut a_cut(int planes, size_t m, size_t np, size_t batch) { return cut_for(planes, m, m, np / kStepK, batch, true, 0, 3, kMaxSplits); }
inline Cut b_cut(int planes, size_t m, size_t mp, size_t batch) { return cut_for(planes, m, m, mp / kStepK, batch, true, 0, 3, 1); }
inline Cut x_cut(int planes, size_t m, size_t n, size_t mp, size_t batch) { return cut_for(planes, m, n, mp / kStepK, batch, false, 0, 3, 1); }

// ---- the gated feed-forward block's forward ----------------------------------

// Paired tiles: a wave holds both projections of the same columns, so a tile has
// half its side of them.  There are 128 x 128, with two buffers and with three
// (indexes of kTiles), and 256 x 256; up to 64 tokens take kFlat.
constexpr int kFlat = -1, kPairSmall = 1, kPairLarge = 3, kPairDeep = 4;
constexpr double kFlatStep = 0.45;

inline size_t pair_tiles(int tile, size_t tokens, size_t hidden) { return tiles_of(1, tile, tokens, 2 * hidden, 1, false); }
// With at most one tile to a unit the three buffers of kPairDeep, else two tiles to
// a unit: 1024 x 4096 x 1408 39 us, with two buffers 62; 128 x 4096 x 11264 48 and 67.
inline int pair_small(size_t runs) { return runs <= 256 ? kPairDeep : kPairSmall; }

// us of a forward, a fit to 932 sizes in every shape (65 to 16384 tokens, dim 128 to
// 6144, hidden 125 to 6144, half of them also with the projections saved; operands in
// the caches): the tile so chosen takes 0.6 % more than the best of them in the mean.
// A step of a tile, several on a unit one after another: 256 x 256 1.45, alone 1.15
// (the clock is higher then); two of 128 x 128 side by side 0.9, one 0.73, a fifth
// more where rows begin between cache lines; with three buffers 0.41.  Their ends 16,
// 3 and 6, between those of calls that save the projections and of those that do not.
// A join: 3 and its bytes at 5 TB/s.  The 256 tile first, then the cheaper 128: 2048 x
// 1024 x 4352 65 us, 54; 1536 x 1024 x 5632 66, 54; but 1536 x 4096 x 2816 92, 112.
inline double pair_us(int tile, size_t tokens, size_t dim, size_t hidden, uint32_t splits)
{
    const size_t units = (pair_tiles(tile, tokens, hidden) * splits + 255) / 256, steps = (dim + kStepK - 1) / kStepK;
    const double per = (double)((steps + splits - 1) / splits);
    const bool between = dim % 8 == 0 && dim % 64 != 0;  // other rows are copied to whole lines
    double us = tile == kPairLarge ? per * (units == 1 ? 1.15 : 1.45 * units) + 16.0 * units
                : tile == kPairDeep ? per * (units == 1 ? 0.41 : 0.5 * units) + 6.0 * units
                                    : per * (between ? 1.2 : 1.0) * (units / 2 * 0.9 + units % 2 * 0.73) + 3.0 * units;
    if (splits > 1) us += 3.0 + 2.0 * splits * 2 * tokens * hidden * 4 / 5e6;
    return us;
}

// The forward's tile and the runs of its k.  Few tiles, of a rank's share of the
// hidden columns say, leave units idle that a split puts to work.  Flat: kFlatStep us
// a step of 64 for a tile (1 x 4096 x 1408 in one piece 32 us), two tiles to a unit,
// the weights' bytes at 4.5 TB/s, and a join as in product_us.  So 1 x 4096 x 5632 is
// split (25 us, in one piece 33) and 1 x 4096 x 11264 is not.
inline Cut ffn_cut(size_t tokens, size_t dim, size_t hidden)
{
    const size_t steps = (dim + kStepK - 1) / kStepK;
    if (tokens <= 64) {
        const size_t tiles = (hidden + 63) / 64;
        const double bytes = 4.0 * dim * hidden / 4.5e6;
        Cut best{kFlat, 1};
        double time = 0;
        for (uint32_t s = 1; s <= kMaxSplits && (s == 1 || s * 2 <= steps); ++s) {
            double sum = (tiles * s + 511) / 512 * ((steps + s - 1) / s) * kFlatStep;
            sum = sum > bytes ? sum : bytes;
            if (s > 1) sum += 4.0 + 2.0 * s * tokens * 2 * hidden * 4 / 6e6;
            if (s == 1 || sum < time) best.splits = s, time = sum;
        }
        return best;
    }
    Cut best{kPairLarge, 1};
    double time = pair_us(kPairLarge, tokens, dim, hidden, 1);
    const size_t tiles = pair_tiles(kPairSmall, tokens, hidden);
    for (uint32_t s = 1; s <= kMaxSplits && may_split(tiles, steps, s); ++s) {
        const int tile = pair_small(tiles * s);
        const double us = pair_us(tile, tokens, dim, hidden, s);
        if (us < time) best = {tile, s}, time = us;
    }
    return best;
}

}  // namespace dev
}  // namespace ar
