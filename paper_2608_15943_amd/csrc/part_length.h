// How long the parts of items are where their number is given (arithmetic alone, for device and host).
//
// Items of t tiles each cut into ceil(t / L) parts make at most (all tiles) / L + items of them: no more than `jobs` where
// L = ceil(tiles / (jobs - items)).
#pragma once

namespace kvp {

constexpr int kWholeItems = 1 << 30;      // a length that cuts nothing

// L for `items` items of `tiles` tiles together (none: 1); the sums may be rounded, in 32 bits and in any order.
constexpr int part_length(int jobs, float items, float tiles) {
    const float room = (float)jobs - items;
    return room < 1.f ? kWholeItems : (int)__builtin_fmaxf(1.f, __builtin_fminf(__builtin_ceilf(tiles * 1.00001f / room), 1e9f));
}

constexpr int parts_of(int tiles, int length) { return (tiles + length - 1) / length; }

}  // namespace kvp
