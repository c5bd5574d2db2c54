// Thousands of random page allocator calls (reserve, release, fork, own, trim, compact), arguments that are none among them,
// with every count checked against the table; built and run under the sanitizers by tests/test_pager_sanitizers.py.
#include <cstdio>
#include <map>
#include <random>
#include <vector>

#include "kvpipe.h"
#include "status.h"

namespace kvp {
char* last_error_buffer() {
    static char buf[512];
    return buf;
}
}  // namespace kvp

static int g_fail = 0;
#define CHECK(c)                                                        \
    do {                                                                \
        if (!(c)) {                                                     \
            std::fprintf(stderr, "line %d: %s\n", __LINE__, #c);        \
            ++g_fail;                                                   \
        }                                                               \
    } while (0)

int main() {
    std::mt19937_64 rng(20261209);
    for (int trial = 0; trial < 30; ++trial) {
        const int n_pages = 1 + (int)(rng() % 200), seqs = 1 + (int)(rng() % 12), width = 1 + (int)(rng() % 30);
        kvp_pager* p = nullptr;
        CHECK(kvp_pager_create(n_pages, seqs, width, &p) == KVP_OK);
        std::vector<int32_t> ids(seqs), rows((size_t)seqs * width);
        for (int i = 0; i < seqs; ++i) ids[i] = i;
        for (int op = 0; op < 3000; ++op) {
            auto seq = [&] { return (int)(rng() % (seqs + 2)) - 1; };
            auto pos = [&] { return (int)(rng() % (64 * width + 200)) - 1; };
            const int room = (int)(rng() % 6);
            std::vector<int32_t> src(room), dst(room);     // as large as the call may fill them
            int n = 0, rc = KVP_OK;
            switch (rng() % 7) {
                case 0: case 1: rc = kvp_pager_reserve(p, seq(), pos()); break;
                case 2: rc = kvp_pager_release(p, seq()); break;
                case 3: rc = kvp_pager_fork(p, seq(), seq(), pos()); break;
                case 4: rc = kvp_pager_own(p, seq(), pos(), rng() % 9 ? pos() : 0x7FFFFFFF, src.data(), dst.data(), room, &n); break;
                case 5: rc = kvp_pager_trim(p, seq(), pos(), rng() % 9 ? pos() : 0x7FFFFFFF); break;
                default: rc = kvp_pager_compact(p, src.data(), dst.data(), room, &n); break;
            }
            CHECK(rc == KVP_OK || rc == KVP_E_CAPACITY || rc == KVP_E_INVALID_ARG || rc == KVP_E_STATE);
            CHECK(n >= 0 && n <= room);
            for (int i = 0; i < n; ++i)
                CHECK(src[i] >= 0 && src[i] < n_pages && dst[i] >= 0 && dst[i] < n_pages && src[i] != dst[i]);
            if (op % 31) continue;
            int free_pages = -1;
            CHECK(kvp_pager_free_pages(p, &free_pages) == KVP_OK);
            CHECK(kvp_pager_rows(p, ids.data(), seqs, rows.data()) == KVP_OK);
            std::map<int32_t, int> held;
            for (int32_t v : rows) {
                CHECK(v >= -1 && v < n_pages);
                if (v >= 0) ++held[v];
            }
            CHECK((int)held.size() + free_pages == n_pages);
        }
        // Everything comes back, each page once.
        for (int s = 0; s < seqs; ++s) CHECK(kvp_pager_release(p, s) == KVP_OK);
        int free_pages = -1;
        CHECK(kvp_pager_free_pages(p, &free_pages) == KVP_OK && free_pages == n_pages);
        kvp_pager_destroy(p);
    }
    if (g_fail) return 1;
    std::printf("pager checks passed\n");
    return 0;
}
