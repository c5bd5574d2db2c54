// The lengths of parts over thousands of calls, empty ones among them: never more parts than there is room for; built and
// run under the sanitizer by tests/test_parts_host.py.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "part_length.h"

int main() {
    std::mt19937_64 rng(20261210);
    auto pick = [&](double lo, double hi) { return (int)(lo * std::pow(hi / lo, (rng() >> 11) * 0x1p-53)); };
    for (int call = 0; call < 20000; ++call) {
        const int jobs = pick(16, 4096), B = pick(1, 300);
        // Sequences of any number of items, of any number of tiles; some, or all, have none.  Items leave room, as the launch sees to.
        std::vector<int> items(B), tiles(B);
        int left = (int)(rng() % jobs);
        float n[64] = {}, t[64];
        unsigned long long lane[64] = {};      // summed as the device does: by lanes, then pairwise
        for (int b = 0; b < B; ++b) {
            const bool none = call % 7 == 0 || rng() % 3 == 0;
            items[b] = none ? 0 : std::min(left, pick(1, jobs));
            tiles[b] = items[b] ? pick(1, 1 << 24) : 0;
            left -= items[b];
            n[b % 64] += (float)items[b];
            lane[b % 64] += (unsigned long long)items[b] * tiles[b];
        }
        for (int i = 0; i < 64; ++i) t[i] = (float)lane[i];
        for (int k = 32; k; k /= 2)
            for (int i = 0; i < k; ++i) n[i] += n[i + k], t[i] += t[i + k];
        const int length = kvp::part_length(jobs, n[0], t[0]);
        long long parts = 0;
        for (int b = 0; b < B; ++b) parts += (long long)items[b] * kvp::parts_of(tiles[b], length);
        if (length < 1 || parts > jobs) {
            std::fprintf(stderr, "call %d: jobs %d, length %d, parts %lld\n", call, jobs, length, parts);
            return 1;
        }
    }
    // Offsets that give rows to several sequences can make more items than the launch takes them for: nothing is cut.
    if (kvp::part_length(512, 512.f, 1e6f) != kvp::kWholeItems || kvp::part_length(512, 1e9f, 1e12f) != kvp::kWholeItems) return 2;
    std::printf("parts checks passed\n");
    return 0;
}
