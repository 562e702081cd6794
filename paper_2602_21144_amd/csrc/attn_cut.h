// Arithmetic of the prompt attention's plan, without a device type in it: it runs in the plan kernel and, compiled for
// the host, in the tests at sizes that no GPU call would reach.
#pragma once
#include <cstdint>

namespace ssm {

// Tiles of a sequence of m rows (token, query head): below 2^23 within the limits of a call
constexpr int32_t tiles_of_rows(int32_t m, int32_t heads, int32_t tile_rows) {
    return (int32_t)(((int64_t)m * heads + tile_rows - 1) / tile_rows);
}
// Sums of tiles stop at this many, more than any call has room for (2^22 and 2^15 of them): sequences whose rows overlap,
// as a program's mistake leaves them, would add up past 32 bits. Sums stay in order, and those below it exact.
constexpr int32_t kManyTiles = 1 << 29;
constexpr int32_t add_tiles(int32_t a, int32_t b) { return a + b < kManyTiles ? a + b : kManyTiles; }


// Steps of the longest item: a place's share of all steps, by the heads that each is taken for, and no less than
// min_steps. The share passes 32 bits where many rows lie behind a long cache (2^18 rows of 32 heads behind 2^30 tokens);
// it stops above the longest tile's steps, which is then not cut.
constexpr int32_t kManySteps = 1 << 25;   // a tile has up to 2^30 / 64 + 1
constexpr int32_t longest_item(uint64_t steps, int32_t heads, int32_t places, int32_t min_steps) {
    const uint64_t share = (steps * (uint64_t)heads + (uint64_t)places - 1) / (uint64_t)places;
    const int32_t most = share < (uint64_t)kManySteps ? (int32_t)share : kManySteps;
    return most < min_steps ? min_steps : most;
}
// A tile of `steps` in pieces of `len` steps (the last one may be shorter), none above `most`
struct TileCut { int32_t pieces, len; };
constexpr TileCut cut_tile(int32_t steps, int32_t most) {
    TileCut c{steps > most ? (steps + most - 1) / most : 1, 0};
    c.len = (steps + c.pieces - 1) / c.pieces;
    if (c.pieces > 1) c.pieces = (steps + c.len - 1) / c.len;
    return c;
}
// The bin of an item of `len` steps: 0 holds the longest
constexpr int32_t item_bin(int32_t len, int32_t most, int32_t bins) {
    return bins - 1 - (int32_t)((uint32_t)len * (uint32_t)bins / (uint32_t)(most + 1));
}

}  // namespace ssm
