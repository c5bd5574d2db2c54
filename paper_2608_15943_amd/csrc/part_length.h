// How long the parts of items are where their number is given (arithmetic alone, for device and host).
//
// Items of t tiles each cut into ceil(t / L) parts make at most (all tiles) / L + items of them: no more than `jobs` where
// L = ceil(tiles / (jobs - items)).
#pragma once

namespace kvp {

constexpr int kWholeItems = 1 << 30;      // a length that cuts nothing

// L for `items` items of `tiles` tiles together; the sums may be rounded, in 32 bits and in any order.
constexpr int part_length(int jobs, float items, float tiles) {
    const float room = (float)jobs - items;
    if (room < 1.f) return kWholeItems;
    const float x = tiles * 1.00001f / room;
    if (x >= 1e9f) return 1000000000;
    const int down = (int)x, n = down + ((float)down < x);
    return n > 0 ? n : 1;                 // no rows at all: no tiles either
}

constexpr int parts_of(int tiles, int length) { return (tiles + length - 1) / length; }

}  // namespace kvp
