// Host-side page allocator for paged KV storage.  A page is 64 positions of one
// sequence; the same page index is used in every producer's pool, so one table row per
// sequence serves all producers (they store the same positions, Eq. 3).  Sharing halves
// (or quarters) the producers, hence the bytes per page index, hence the pages a fixed
// amount of HBM holds: that is the capacity side of KV sharing.
//
// A page may be held by several sequences (a shared prefix, after a fork): refs counts them, and a page
// is free when nobody holds it.  A row may have holes (-1) where a window has left pages behind, or where
// tokens were not accepted; who writes there gets pages again (kvp_pager_own).
//
// Pure host code: no device memory is touched; the caller copies table rows to the device, and pages
// (kvp_copy_pages) where a call here says so.
#include <algorithm>
#include <cstdint>
#include <functional>
#include <new>
#include <vector>

#include "kvpipe.h"
#include "status.h"

using kvp::fail;
using kvp::ok;

struct kvp_pager {
    int n_pages, max_seqs, max_pages;
    std::vector<int32_t> table;   // [max_seqs][max_pages], -1 where unmapped
    std::vector<int32_t> held;    // entries of a row in use, holes among them
    std::vector<int32_t> free;    // free pages; the back is handed out next
    std::vector<int32_t> refs;    // [n_pages] sequences that hold the page
    std::vector<int32_t> moved;   // [n_pages] scratch of kvp_pager_compact
    int32_t* row(int seq) { return table.data() + (size_t)seq * max_pages; }
    int32_t take() {
        const int32_t page = free.back();
        free.pop_back();
        refs[page] = 1;
        return page;
    }
    void drop(int32_t& entry) {
        if (entry >= 0 && --refs[entry] == 0) free.push_back(entry);   // within the capacity: at most n_pages
        entry = -1;
    }
};

namespace {

int check_seq(const kvp_pager* p, int seq, const char* who) {
    if (!p) return fail(KVP_E_INVALID_ARG, "%s: NULL pager", who);
    if (seq < 0 || seq >= p->max_seqs) return fail(KVP_E_INVALID_ARG, "%s: sequence %d out of range", who, seq);
    return KVP_OK;
}

constexpr int kPageTokens = 64;

}  // namespace

extern "C" int kvp_pager_create(int n_pages, int max_seqs, int max_pages_per_seq, kvp_pager** out) {
    if (!out) return fail(KVP_E_INVALID_ARG, "kvp_pager_create: NULL out");
    *out = nullptr;
    if (n_pages < 1 || max_seqs < 1 || max_pages_per_seq < 1)
        return fail(KVP_E_INVALID_ARG, "kvp_pager_create: sizes must be >= 1");
    if ((int64_t)max_seqs * max_pages_per_seq > (int64_t)1 << 31)
        return fail(KVP_E_INVALID_ARG, "kvp_pager_create: table of %d x %d entries is too large", max_seqs,
                    max_pages_per_seq);
    kvp_pager* p = nullptr;
    try {
        p = new kvp_pager;
        p->n_pages = n_pages;
        p->max_seqs = max_seqs;
        p->max_pages = max_pages_per_seq;
        p->table.assign((size_t)max_seqs * max_pages_per_seq, -1);
        p->held.assign(max_seqs, 0);
        p->free.resize(n_pages);
        p->refs.assign(n_pages, 0);
        p->moved.resize(n_pages);
    } catch (const std::bad_alloc&) {
        delete p;
        return fail(KVP_E_CAPACITY, "kvp_pager_create: out of host memory");
    }
    for (int i = 0; i < n_pages; ++i) p->free[i] = n_pages - 1 - i;   // page 0 first
    *out = p;
    return ok();
}

extern "C" void kvp_pager_destroy(kvp_pager* p) { delete p; }

extern "C" int kvp_pager_reserve(kvp_pager* p, int seq, int n_tokens) {
    if (const int rc = check_seq(p, seq, "kvp_pager_reserve")) return rc;
    if (n_tokens < 0) return fail(KVP_E_INVALID_ARG, "kvp_pager_reserve: n_tokens < 0");
    const int64_t need = ((int64_t)n_tokens + kPageTokens - 1) / kPageTokens;
    if (need > p->max_pages)
        return fail(KVP_E_CAPACITY, "kvp_pager_reserve: %d tokens need %lld pages, a row holds %d", n_tokens,
                    (long long)need, p->max_pages);
    const int have = p->held[seq], last = std::min((int)need, have) - 1;
    int32_t* row = p->row(seq);
    if (last >= 0 && row[last] < 0)
        return fail(KVP_E_CAPACITY, "kvp_pager_reserve: positions from %d on of sequence %d were trimmed (kvp_pager_own maps them)",
                    last * kPageTokens, seq);
    if (need <= have) return ok();
    const int add = (int)need - have;
    if ((size_t)add > p->free.size())
        return fail(KVP_E_CAPACITY, "kvp_pager_reserve: %d more pages needed, %zu free", add, p->free.size());
    for (int j = have; j < (int)need; ++j) row[j] = p->take();
    p->held[seq] = (int)need;
    return ok();
}

extern "C" int kvp_pager_release(kvp_pager* p, int seq) {
    if (const int rc = check_seq(p, seq, "kvp_pager_release")) return rc;
    int32_t* row = p->row(seq);
    for (int j = p->held[seq] - 1; j >= 0; --j) p->drop(row[j]);   // the sequence's first page comes out first again
    p->held[seq] = 0;
    return ok();
}

extern "C" int kvp_pager_fork(kvp_pager* p, int from, int to, int n_tokens) {
    if (const int rc = check_seq(p, from, "kvp_pager_fork")) return rc;
    if (const int rc = check_seq(p, to, "kvp_pager_fork")) return rc;
    if (from == to || n_tokens < 0) return fail(KVP_E_INVALID_ARG, "kvp_pager_fork: from == to, or n_tokens < 0");
    if (p->held[to]) return fail(KVP_E_STATE, "kvp_pager_fork: sequence %d holds pages", to);
    const int64_t need = ((int64_t)n_tokens + kPageTokens - 1) / kPageTokens;
    if (need > p->held[from])
        return fail(KVP_E_CAPACITY, "kvp_pager_fork: sequence %d has no pages for %d tokens", from, n_tokens);
    const int32_t* src = p->row(from);
    int32_t* dst = p->row(to);
    for (int j = 0; j < (int)need; ++j) {
        dst[j] = src[j];
        if (src[j] >= 0) ++p->refs[src[j]];
    }
    p->held[to] = (int)need;
    return ok();
}

extern "C" int kvp_pager_own(kvp_pager* p, int seq, int from, int to, int32_t* src, int32_t* dst, int max_pairs, int* n) {
    if (const int rc = check_seq(p, seq, "kvp_pager_own")) return rc;
    if (!n || max_pairs < 0 || (max_pairs && (!src || !dst)) || from < 0 || to < from)
        return fail(KVP_E_INVALID_ARG, "kvp_pager_own: NULL argument, or a range that is none");
    *n = 0;
    int32_t* row = p->row(seq);
    const int j0 = from / kPageTokens;
    const int j1 = from == to ? j0 : std::min<int64_t>(((int64_t)to + kPageTokens - 1) / kPageTokens, p->held[seq]);
    // Rows at `from` follow the position in front of it: a page for theirs alone would be no use.
    if (j0 < j1 && row[j0] < 0 && from > 0 && row[(from - 1) / kPageTokens] < 0)
        return fail(KVP_E_CAPACITY, "kvp_pager_own: sequence %d has no page for position %d", seq, from - 1);
    // Holes from the row's beginning up to its first page are a window's and stay.
    int first = 0, pairs = 0, gone = 0;
    while (first < p->held[seq] && row[first] < 0) ++first;
    if (first == p->held[seq]) first = 0;
    for (int j = j0; j < j1; ++j) {
        pairs += row[j] >= 0 && p->refs[row[j]] > 1;
        gone += row[j] < 0 && j >= first;
    }
    if ((size_t)pairs + gone > p->free.size())
        return fail(KVP_E_CAPACITY, "kvp_pager_own: %d pages needed, %zu free", pairs + gone, p->free.size());
    if (pairs > max_pairs) return fail(KVP_E_CAPACITY, "kvp_pager_own: %d pages to copy, room for %d", pairs, max_pairs);
    for (int j = j0; j < j1; ++j)
        if (row[j] < 0) {
            if (j >= first) row[j] = p->take();
        } else if (p->refs[row[j]] > 1) {
            src[*n] = row[j];
            --p->refs[row[j]];
            row[j] = dst[*n] = p->take();
            ++*n;
        }
    return ok();
}

extern "C" int kvp_pager_trim(kvp_pager* p, int seq, int from, int to) {
    if (const int rc = check_seq(p, seq, "kvp_pager_trim")) return rc;
    if (from < 0) return fail(KVP_E_INVALID_ARG, "kvp_pager_trim: from < 0");
    if (to <= from) return ok();
    int32_t* row = p->row(seq);
    const int j0 = std::min<int64_t>(((int64_t)from + kPageTokens - 1) / kPageTokens, p->held[seq]);
    const int j1 = std::min(to / kPageTokens, p->held[seq]);
    for (int j = j1 - 1; j >= j0; --j) p->drop(row[j]);
    return ok();
}

extern "C" int kvp_pager_compact(kvp_pager* p, int32_t* src, int32_t* dst, int max_pairs, int* n) {
    if (!p || !n || max_pairs < 0 || (max_pairs && (!src || !dst)))
        return fail(KVP_E_INVALID_ARG, "kvp_pager_compact: NULL argument, or max_pairs < 0");
    *n = 0;
    // The free pages, highest first: the lowest is handed out next, here and by what follows.
    std::sort(p->free.begin(), p->free.end(), std::greater<int32_t>());
    const int used = p->n_pages - (int)p->free.size();
    for (int page = p->n_pages - 1; page >= used && *n < max_pairs; --page)
        if (p->refs[page] > 0) {
            src[*n] = page;
            dst[*n] = p->free.back();       // below `used`: as many are free there as are held above
            p->free.pop_back();
            ++*n;
        }
    if (*n == 0) return ok();
    for (int i = 0; i < p->n_pages; ++i) p->moved[i] = i;
    for (int i = 0; i < *n; ++i) {
        p->moved[src[i]] = dst[i];
        p->refs[dst[i]] = p->refs[src[i]];
        p->refs[src[i]] = 0;
        p->free.push_back(src[i]);
    }
    std::sort(p->free.begin(), p->free.end(), std::greater<int32_t>());
    for (int s = 0; s < p->max_seqs; ++s) {
        int32_t* row = p->row(s);
        for (int j = 0; j < p->held[s]; ++j)
            if (row[j] >= 0) row[j] = p->moved[row[j]];
    }
    return ok();
}

extern "C" int kvp_pager_free_pages(const kvp_pager* p, int* n) {
    if (!p || !n) return fail(KVP_E_INVALID_ARG, "kvp_pager_free_pages: NULL argument");
    *n = (int)p->free.size();
    return ok();
}

extern "C" int kvp_pager_rows(const kvp_pager* p, const int32_t* seqs, int B, int32_t* out) {
    if (!p || !seqs || !out || B < 0) return fail(KVP_E_INVALID_ARG, "kvp_pager_rows: NULL argument or B < 0");
    for (int i = 0; i < B; ++i)
        if (seqs[i] < 0 || seqs[i] >= p->max_seqs)
            return fail(KVP_E_INVALID_ARG, "kvp_pager_rows: sequence %d out of range", seqs[i]);
    for (int i = 0; i < B; ++i) {
        const int32_t* row = p->table.data() + (size_t)seqs[i] * p->max_pages;
        for (int j = 0; j < p->max_pages; ++j) out[(size_t)i * p->max_pages + j] = row[j];
    }
    return ok();
}
