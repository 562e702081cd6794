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

}  // namespace ssm
