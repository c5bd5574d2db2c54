// Attention of a call's new rows over the 8-bit paged cache: one new token a sequence, a few, or
// a whole prompt; row i of sequence b sits at position len_b + i and sees positions [0, len_b + i].
//
// The rows of a sequence and the r = a / g query heads of a K/V head are the columns of one
// product: an item is m = 16 NB / r rows of a sequence with the r heads of a K/V head, and a wave
// runs over the item's 64-position tiles (a page each) once, with the running maximum and sum of
// the softmax, without LDS or barriers: K and V go from memory to registers in 16-byte runs, are
// widened to bf16 there (exactly: e4m3 has 4 significant bits) and multiplied on
// v_mfma_f32_16x16x32_bf16.
//
//   S^T = K Q^T  Row rho of score block tb is position 16 (rho / 4) + 4 tb + rho % 4 of the tile, so
//                that lane group grp ends with positions 16 grp .. 16 grp + 15: one scale block, and
//                the run that the second product sums over.  The K scale multiplies a lane's
//                scores, one factor for all of them.
//   O^T += V^T P^T  The V scale, a power of two, goes into the exponent of P before P is rounded to
//                bf16 (8 bits); the sum of the weights is taken from the rounded P, so that its
//                rounding cancels where it is common.
//
// Work: the tiles of all items in one list, in the order (sequence, K/V head, block of rows, tile),
// which W waves share evenly: an item that begins and ends with one wave is written by it, the others
// leave their pieces (running maximum, sum, unnormalised O) to a second kernel.  Where there are many
// more items than waves they run one by one instead, the longest first.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "fp8_cache.h"

namespace kvp {
namespace {

constexpr int D = kHead, TILE = kPage;
constexpr int PSTRIDE = D + 4;    // O[128], m, l, pad
constexpr float kLazy = 8.0f;     // the running maximum follows once it is 2^8 behind

// 8 codes (two words) as bf16.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

struct KTile {
    u32x4 k[4][2];     // [score block][64-dimension half]
    float s;           // scale of the lane group's 16 positions
};
struct VTile {
    u32x4 v[8];        // [16-dimension block]
    float s;
};

struct AttnArgs {
    NewRows r;
    const uint16_t* q;
    const uint8_t* kc;
    const uint8_t* vc;
    const float* sc;
    uint16_t* out;
    float* part;       // [2 waves][cols][PSTRIDE]: slot 2 w: wave w's piece of an item that began before it,
                       // 2 w + 1: of one that begins with it and goes on
    int a, g;
    int m, cols;       // rows of an item, columns that they make
    float scale_log2;
};

// sum of floor((A i + B) / M) over 0 <= i < N, by Euclid's steps.
__device__ __forceinline__ uint32_t floor_sum(uint32_t N, uint32_t M, uint32_t A, uint32_t B) {
    uint32_t s = 0;
    while (N) {
        s += (uint32_t)((uint64_t)N * (N - 1) / 2) * (A / M) + N * (B / M);
        A %= M;
        B %= M;
        const uint32_t y = A * N + B;
        N = y / M;
        B = y % M;
        const uint32_t t = M;
        M = A;
        A = t;
    }
    return s;
}

// Tiles of block c of a sequence, and of its first c blocks; a block without a row that sees anything
// counts one (it writes zeros).
__device__ __forceinline__ int tiles_of(const SeqRows& s, int m, int c) {
    const int last = min((c + 1) * m, s.act) - 1;
    return last < c * m ? 1 : (s.len + last) / TILE + 1;
}
__device__ __forceinline__ uint32_t tiles_before(const SeqRows& s, int m, int c) {
    const int full = min(c, s.act / m);            // blocks whose m rows all see something
    uint32_t n = full + floor_sum(full, TILE, m, s.len + m - 1);
    if (c > full) n += tiles_of(s, m, full) + (c - full - 1);
    return n;
}
__device__ __forceinline__ int blocks_of(const SeqRows& s, int m) { return (s.n + m - 1) / m; }

// The list shared by W waves: wave w starts at tile floor(w T / W).  T < 2^31, W <= 4096.
struct Split {
    uint32_t T, W, q, rem;
    __device__ __forceinline__ Split(uint32_t T_, uint32_t waves) : T(T_), W(min(T_, waves)), q(T_ / max(W, 1u)), rem(T_ % max(W, 1u)) {}
    __device__ __forceinline__ uint32_t start(uint32_t w) const { return w * q + w * rem / W; }
    // The wave that holds tile x: ceil((x + 1) W / T) - 1; exact in double.
    __device__ __forceinline__ uint32_t wave_of(uint32_t x) const {
        return (uint32_t)(((double)(x + 1) * (double)W - 1.0) / (double)T);
    }
};

// 64 sequences at a time, one a lane: their rows, tiles for one K/V head, and the tiles of the list
// before each.
struct Lanes {
    int b0;
    SeqRows s;
    uint32_t n, pre;     // pre: before this lane's sequence
    uint32_t total;      // tiles of the 64
    __device__ __forceinline__ void load(const AttnArgs& A, int b0_, uint32_t base) {
        const int lane = threadIdx.x & 63;
        b0 = b0_;
        s = SeqRows{0, 0, 0, 0};
        n = 0;
        if (b0 + lane < A.r.B) {
            s = seq_rows(A.r, b0 + lane);
            n = tiles_before(s, A.m, blocks_of(s, A.m));
        }
        uint32_t p = n * A.g;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t v = __shfl_up(p, off);
            if (lane >= off) p += v;
        }
        total = __builtin_amdgcn_readlane(p, 63);
        pre = base + p - n * A.g;
    }
    __device__ __forceinline__ SeqRows rows(int w) const {
        return {__builtin_amdgcn_readlane(s.row0, w), __builtin_amdgcn_readlane(s.n, w),
                __builtin_amdgcn_readlane(s.len, w), __builtin_amdgcn_readlane(s.act, w)};
    }
};
__device__ __forceinline__ uint32_t list_tiles(const AttnArgs& A, Lanes& L) {
    uint32_t T = 0;
    for (int b0 = 0; b0 < A.r.B; b0 += 64) {
        L.load(A, b0, T);
        T += L.total;
    }
    return T;
}

// An item and a place in it.
struct Item {
    int b, kvh, c;       // sequence, K/V head, block of rows
    SeqRows s;
    int t, n;            // tile, tiles
};
// The item that holds tile x of the list (x < T).
__device__ __forceinline__ Item find_tile(const AttnArgs& A, Lanes& L, uint32_t x) {
    if (A.r.B > 64) {
        uint32_t base = 0;
        for (int b0 = 0;; b0 += 64) {
            L.load(A, b0, base);
            if (x < base + L.total) break;
            base += L.total;
        }
    }
    Item it;
    // The last lane that begins at or before x and has tiles: those behind it begin later.
    const int w = 63 - __builtin_clzll(__ballot(L.n > 0 && L.pre <= x));
    it.b = L.b0 + w;
    it.s = L.rows(w);
    const uint32_t n = __builtin_amdgcn_readlane(L.n, w);
    uint32_t rem = x - __builtin_amdgcn_readlane(L.pre, w);
    it.kvh = rem / n;
    rem %= n;
    int lo = 0, hi = blocks_of(it.s, A.m) - 1;         // the last block with tiles_before <= rem
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (tiles_before(it.s, A.m, mid) <= rem)
            lo = mid;
        else
            hi = mid - 1;
    }
    it.c = lo;
    it.t = rem - (lo ? tiles_before(it.s, A.m, lo) : 0);
    it.n = tiles_of(it.s, A.m, lo);
    return it;
}

// LIST: the wave's share of the list; else item blockIdx.x, counted from the last.
template <int NB, bool LIST>
__global__ __launch_bounds__(64, NB == 1 ? 3 : 2) void attention_kernel(AttnArgs A) {
    const int lane = threadIdx.x, col = lane & 15, grp = lane >> 4;
    const int r = A.a / A.g;
    Item it;
    Lanes L;
    uint32_t w = 0, left;                       // tiles left of the wave's share
    if constexpr (LIST) {
        const Split sp(list_tiles(A, L), gridDim.x);
        if (blockIdx.x >= sp.W) return;
        w = xcd_remap(blockIdx.x, sp.W);
        const uint32_t x = sp.start(w);
        left = sp.start(w + 1) - x;
        it = find_tile(A, L, x);
    } else {
        // K/V heads change fastest: with 8 of them each XCD reads one of them only.
        int first;
        const int x = blockIdx.x / A.g;
        auto blocks = [&](const SeqRows& s) { return blocks_of(s, A.m); };
        if (!find_item(A.r, x, blocks, &it.b, &it.s, &first)) return;
        it.c = blocks_of(it.s, A.m) - 1 - (x - first);
        it.kvh = blockIdx.x % A.g;
        it.t = 0;
        it.n = tiles_of(it.s, A.m, it.c);
        left = it.n;
    }

    // Columns: head tj of row tc of a block; a lane's column of block cb.
    int tc[NB], tj[NB];
    bool valid[NB];
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) {
        const int c = 16 * cb + col;
        valid[cb] = c < A.cols;
        tc[cb] = valid[cb] ? c / r : 0;
        tj[cb] = valid[cb] ? c % r : 0;
    }
    // The last position that a column sees, -1 where there is none.
    auto limit = [&](const Item& i, int cb) {
        const int t = i.c * A.m + tc[cb];
        return valid[cb] && t < i.s.act ? i.s.len + t : -1;
    };
    // Contraction order of S: step ks of lane group grp holds dimensions 64 (ks / 2) + 16 grp +
    // 8 (ks % 2) .. + 7, the order of the K codes' 16-byte runs.
    auto load_q = [&](const Item& i, bf16x8 (&qf)[NB][4]) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            const bool real = limit(i, cb) >= 0;
            const size_t row = i.s.row0 + (real ? i.c * A.m + tc[cb] : 0);
            const uint16_t* p = A.q + (row * A.a + i.kvh * r + tj[cb]) * D + 16 * grp;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                u32x4 v = u32x4{0, 0, 0, 0};
                if (real) v = *(const u32x4*)(p + 64 * (ks >> 1) + 8 * (ks & 1));
                qf[cb][ks] = as_bf16x8(v);
            }
        }
    };
    // The wave keeps 64 entries of a table row, so that one dependent load serves 64 tiles.
    int pb = -1, pc = -1, pgv = 0;
    auto page_at = [&](const Item& i) {
        if (i.b != pb || (i.t >> 6) != pc) {
            pb = i.b;
            pc = i.t >> 6;
            const int e = 64 * pc + lane;
            pgv = e < A.r.stride ? A.r.pt[(size_t)i.b * A.r.stride + e] : 0;
        }
        const int pg = min(max(__builtin_amdgcn_readlane(pgv, i.t & 63), 0), A.r.n_pages - 1);
        return (size_t)i.kvh * A.r.n_pages + pg;
    };
    const int koff = (16 * (col >> 2) + (col & 3)) * D + 16 * grp, voff = grp * kBlkBytes + col * kBlk;
    auto load_k = [&](size_t at, KTile& k) {
        const uint8_t* p = A.kc + at * kPageBytes8 + koff;
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int j = 0; j < 2; ++j) k.k[tb][j] = *(const u32x4*)(p + 4 * tb * D + 64 * j);
        k.s = A.sc[at * 2 * kPageBlks + grp];
    };
    auto load_v = [&](size_t at, VTile& v) {
        const uint8_t* p = A.vc + at * kPageBytes8 + voff;
#pragma unroll
        for (int db = 0; db < 8; ++db) v.v[db] = *(const u32x4*)(p + 16 * db * kBlk);
        v.s = A.sc[at * 2 * kPageBlks + kPageBlks + grp];
    };

    bf16x8 qf[NB][4];
    f32x4 o[NB][8];
    float m_run[NB], l_run[NB];
    int lim[NB], all = 0, last = 0;
    // Begins an item (qf loaded).
    auto begin = [&](const Item& i) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            lim[cb] = limit(i, cb);
            m_run[cb] = kNoScore;
            l_run[cb] = 0.f;
#pragma unroll
            for (int db = 0; db < 8; ++db) o[cb][db] = f32x4{};
        }
        // Positions up to `all` every row sees, past `last` none does.
        const int rows = min(i.s.act - i.c * A.m, A.m);
        all = rows > 0 ? i.s.len + i.c * A.m : -1;
        last = rows > 0 ? i.s.len + i.c * A.m + rows - 1 : -1;
    };

    KTile kt;
    VTile vt;
    f32x4 sc[NB][4];
    bf16x8 pb16[NB][2];
    auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const bf16x8 kf = widen(kt.k[tb][ks >> 1][2 * (ks & 1)], kt.k[tb][ks >> 1][2 * (ks & 1) + 1]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) sc[cb][tb] = mfma16x16x32(kf, qf[cb][ks], ks ? sc[cb][tb] : f32x4{});
            }
    };
    // Lane (col, grp) holds its column's scores at positions p0 + 4 tb + i.  edge: some column does not
    // see all of the tile (one branch for all of it: two copies of this code would not fit the registers).
    auto softmax = [&](bool edge, int p0, float ks) __attribute__((always_inline)) {
        // P 2^e for a V scale of 2^e.
        const int e = (int)(__float_as_uint(vt.s) >> 23) - 127;
        const float vexp = vt.s == vt.s ? (float)e : vt.s;
        const float vinv = vt.s == vt.s ? __uint_as_float((uint32_t)(127 - e) << 23) : 1.f;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            if (edge) {
#pragma unroll
                for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (p0 + 4 * tb + i > lim[cb]) sc[cb][tb][i] = -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[cb][tb][i]);
            const float mt = pair32_max(pair16_max(mx * ks));
            if (__any(mt > m_run[cb] + kLazy)) {
                const float m_new = fmaxf(m_run[cb], mt);
                const float alpha = __builtin_amdgcn_exp2f(m_run[cb] - m_new);
                m_run[cb] = m_new;
                l_run[cb] *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db) o[cb][db] *= alpha;
            }
            const float sub = vexp - m_run[cb];
            uint32_t pw[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                pw[i] = pack2bf(__builtin_amdgcn_exp2f(fmaf(sc[cb][i >> 1][2 * (i & 1)], ks, sub)),
                                __builtin_amdgcn_exp2f(fmaf(sc[cb][i >> 1][2 * (i & 1) + 1], ks, sub)));
            if (edge) {
                // Whatever a hidden position's scales hold (NaN perhaps), it weighs nothing.
                const int n = lim[cb] + 1 - p0;       // positions of the lane's 16 that the column sees
#pragma unroll
                for (int i = 0; i < 8; ++i) pw[i] &= n > 2 * i + 1 ? 0xFFFFFFFFu : n > 2 * i ? 0xFFFFu : 0u;
            }
            float lt = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                lt = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[i]),
                                                     __builtin_bit_cast(bf16x2, 0x3F803F80u), lt, false);
            l_run[cb] += lt * vinv;
            pb16[cb][0] = as_bf16x8(u32x4{pw[0], pw[1], pw[2], pw[3]});
            pb16[cb][1] = as_bf16x8(u32x4{pw[4], pw[5], pw[6], pw[7]});
        }
        if (edge) {
            // Codes past the last position that a column sees (never written, perhaps) must be finite:
            // they count as 0.
            const int n = last + 1 - p0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = n - 4 * i;              // bytes of word i that are seen
                const uint32_t mask = k >= 4 ? 0xFFFFFFFFu : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
#pragma unroll
                for (int db = 0; db < 8; ++db) vt.v[db][i] &= mask;
            }
        }
    };
    auto values = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 vf = widen(vt.v[db][2 * h], vt.v[db][2 * h + 1]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) o[cb][db] = mfma16x16x32(vf, pb16[cb][h], o[cb][db]);
            }
    };

    bool whole = it.t == 0;        // the wave has the item from its first tile on
    load_q(it, qf);
    begin(it);
    {
        const size_t at = page_at(it);
        load_k(at, kt);
        load_v(at, vt);
    }
    for (;;) {
        // The next tile of the share, perhaps in the next item.
        const bool ends = it.t + 1 == it.n;
        bool more = left > 1;
        Item nx = it;
        if (more) {
            ++nx.t;
            if (LIST && ends) {
                nx.t = 0;
                if (++nx.c == blocks_of(nx.s, A.m)) {
                    nx.c = 0;
                    if (++nx.kvh == A.g) {
                        nx.kvh = 0;
                        for (++nx.b; nx.b < A.r.B; ++nx.b) {       // sequences without rows have no tiles
                            if (nx.b - L.b0 == 64) L.load(A, nx.b, 0);
                            if (__builtin_amdgcn_readlane(L.n, nx.b - L.b0)) break;
                        }
                        more = nx.b < A.r.B;
                        if (more) nx.s = L.rows(nx.b - L.b0);
                    }
                }
                nx.n = tiles_of(nx.s, A.m, nx.c);
            }
        }
        const size_t at = more ? page_at(nx) : 0;
        const int t0 = TILE * it.t, p0 = t0 + 16 * grp;
        scores();
        const float ks = kt.s * A.scale_log2;
        __builtin_amdgcn_sched_barrier(0);
        // A part of a tile (and the queries) is requested again as soon as it has been multiplied: 16
        // KB a wave are always under way, without a second set of registers.
        if (more) {
            load_k(at, kt);
            if (LIST && ends) load_q(nx, qf);
        }
        __builtin_amdgcn_sched_barrier(0);
        const bool edge = t0 + TILE - 1 > all;
        // The scales of blocks that no column sees may hold anything.
        if (edge && p0 > last) vt.s = 1.f;
        softmax(edge, p0, edge && p0 > last ? A.scale_log2 : ks);
        __builtin_amdgcn_sched_barrier(0);
        values();
        __builtin_amdgcn_sched_barrier(0);
        if (more) load_v(at, vt);
        if (ends || !more) {
            // O^T block db: lane holds dimensions 16 db + 4 grp + 0..3 of its column.
#pragma unroll
            for (int cb = 0; cb < NB; ++cb) {
                const float l = pair32_sum(pair16_sum(l_run[cb]));
                const int t = it.c * A.m + tc[cb];
                if (!valid[cb] || t >= it.s.n) continue;
                if (whole && ends) {
                    const float inv = 1.f / l;
                    uint16_t* op = A.out + ((size_t)(it.s.row0 + t) * A.a + it.kvh * r + tj[cb]) * D + 4 * grp;
#pragma unroll
                    for (int db = 0; db < 8; ++db) {
                        u32x2 v = {pack2bf(o[cb][db][0] * inv, o[cb][db][1] * inv),
                                   pack2bf(o[cb][db][2] * inv, o[cb][db][3] * inv)};
                        if (lim[cb] < 0) v = u32x2{0, 0};      // sees nothing
                        *(u32x2*)(op + 16 * db) = v;
                    }
                } else if constexpr (LIST) {
                    float* pr = A.part + ((size_t)(2 * w + (whole ? 1 : 0)) * A.cols + 16 * cb + col) * PSTRIDE;
#pragma unroll
                    for (int db = 0; db < 8; ++db) *(f32x4*)(pr + 16 * db + 4 * grp) = o[cb][db];
                    if (grp == 0) {
                        pr[D] = m_run[cb];
                        pr[D + 1] = l;
                    }
                }
            }
            if (LIST && more) {
                whole = true;
                begin(nx);
            }
        }
        if (!more) break;
        it = nx;
        --left;
    }
}

// Where the pieces of an item are joined: waves w0 (from the item's first tile on) .. w0 + np - 1.
struct Pieces {
    uint32_t w0;
    int np;
    __device__ __forceinline__ size_t slot(int i) const { return 2 * (size_t)(w0 + i) + (i == 0 ? 1 : 0); }
};

constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / 64;

// One new row a sequence or a few (an item is a sequence and K/V head): a workgroup a column.  Wave
// v takes pieces v, v + 4, ...: lane i holds the maximum and sum of its i-th, every lane two of the
// 128 dimensions; the waves meet in LDS.
__global__ __launch_bounds__(kJoinThreads) void join_few_kernel(AttnArgs A, int waves) {
    __shared__ float num_s[kJoinWaves][D], m_s[kJoinWaves], den_s[kJoinWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int x = blockIdx.x / A.cols, c = blockIdx.x % A.cols, b = x / A.g, kvh = x % A.g, r = A.a / A.g;
    // The sequence's place in the list.
    Lanes L;
    uint32_t T = 0, n = 0, x0 = 0;
    SeqRows s{};
    for (int b0 = 0; b0 < A.r.B; b0 += 64) {
        L.load(A, b0, T);
        T += L.total;
        if (b >= b0 && b < b0 + 64) {
            s = L.rows(b - b0);
            n = __builtin_amdgcn_readlane(L.n, b - b0);
            x0 = __builtin_amdgcn_readlane(L.pre, b - b0) + kvh * n;
        }
    }
    const int t = c / r;
    if (t >= s.n) return;
    const Split sp(T, waves);
    Pieces pc;
    pc.w0 = __builtin_amdgcn_readfirstlane((int)sp.wave_of(x0));
    pc.np = __builtin_amdgcn_readfirstlane((int)sp.wave_of(x0 + n - 1)) - pc.w0 + 1;
    if (pc.np == 1) return;                       // written by its wave
    const size_t step = (size_t)A.cols * PSTRIDE;
    const float* part = A.part + (size_t)c * PSTRIDE;
    const int mine = (pc.np - wave + kJoinWaves - 1) / kJoinWaves;
    float M = -INFINITY, den = 0.f;
    f32x2 num = {0.f, 0.f};
    for (int s0 = 0; s0 < mine; s0 += 64) {
        const int k = min(mine - s0, 64);
        auto piece = [&](int i) { return part + pc.slot(wave + kJoinWaves * (s0 + i)) * step; };
        float m = -INFINITY, l = 0.f;
        if (lane < k) {
            const float* p = piece(lane);
            m = p[D];
            l = p[D + 1];
        }
        const float Mn = fmaxf(M, wave_max(m)), f = exp2f(M - Mn), wt = exp2f(m - Mn);
        den = den * f + wave_sum(lane < k ? wt * l : 0.f);
        num *= f;
        M = Mn;
        auto add = [&](auto n_t, int i0) __attribute__((always_inline)) {
            constexpr int N = decltype(n_t)::value;
            f32x2 v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = *(const f32x2*)(piece(i0 + i) + 2 * lane);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wt), i0 + i));
                num[0] += w * v[i][0];
                num[1] += w * v[i][1];
            }
        };
        int i = 0;
        for (; i + 8 <= k; i += 8) add(std::integral_constant<int, 8>{}, i);
        for (; i + 4 <= k; i += 4) add(std::integral_constant<int, 4>{}, i);
        for (; i < k; ++i) add(std::integral_constant<int, 1>{}, i);
    }
    *(f32x2*)&num_s[wave][2 * lane] = num;
    if (lane == 0) {
        m_s[wave] = M;
        den_s[wave] = den;
    }
    __syncthreads();
    if (tid >= D) return;
    float Mx = m_s[0];
#pragma unroll
    for (int v = 1; v < kJoinWaves; ++v) Mx = fmaxf(Mx, m_s[v]);
    float ns = 0.f, ds = 0.f;
#pragma unroll
    for (int v = 0; v < kJoinWaves; ++v) {
        const float f = exp2f(m_s[v] - Mx);
        ns += f * num_s[v][tid];
        ds += f * den_s[v];
    }
    A.out[((size_t)(s.row0 + t) * A.a + kvh * r + c % r) * D + tid] = t < s.act ? f2bf(ns / ds) : (uint16_t)0;
}

// Many rows: a workgroup a boundary of the list between two waves, which joins the item that the
// boundary cuts if it is the first to cut it; a wave a column in turn.
__global__ __launch_bounds__(kJoinThreads) void join_many_kernel(AttnArgs A, int waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = A.a / A.g;
    Lanes L;
    const Split sp(list_tiles(A, L), waves);
    const uint32_t w = blockIdx.x + 1;
    if (w >= sp.W) return;
    const uint32_t x = sp.start(w);
    const Item it = find_tile(A, L, x);
    const uint32_t x0 = x - it.t;
    if (it.t == 0 || sp.start(w - 1) > x0) return;
    Pieces pc;
    pc.w0 = w - 1;
    pc.np = sp.wave_of(x0 + it.n - 1) - pc.w0 + 1;
    const size_t step = (size_t)A.cols * PSTRIDE;
    for (int c = wave; c < A.cols; c += kJoinWaves) {
        const int t = it.c * A.m + c / r;
        if (t >= it.s.n) break;
        float M = -INFINITY, den = 0.f;
        f32x2 num = {0.f, 0.f};
        for (int i = 0; i < pc.np; ++i) {
            const float* p = A.part + pc.slot(i) * step + (size_t)c * PSTRIDE;
            const f32x2 v = *(const f32x2*)(p + 2 * lane);
            const float m = p[D], Mn = fmaxf(M, m), f = exp2f(M - Mn), wt = exp2f(m - Mn);
            den = den * f + wt * p[D + 1];
            num[0] = num[0] * f + wt * v[0];
            num[1] = num[1] * f + wt * v[1];
            M = Mn;
        }
        const uint32_t o = t < it.s.act ? pack2bf(num[0] / den, num[1] / den) : 0u;
        *(uint32_t*)(A.out + ((size_t)(it.s.row0 + t) * A.a + it.kvh * r + c % r) * D + 2 * lane) = o;
    }
}

// Two waves a SIMD.
int list_waves(int simds) { return std::min(2 * simds, kMaxDecodeSplits); }

}  // namespace

size_t attention_fp8_floats(int simds) { return (size_t)2 * list_waves(simds) * 32 * PSTRIDE; }

hipError_t attention_fp8(const NewRows& r, int a, int g, const uint16_t* q, const uint8_t* kc, const uint8_t* vc,
                         const float* sc, uint16_t* out, float* part, int simds, hipStream_t st) {
    if (r.B < 1 || r.rows < 1 || r.n_pages < 1 || r.stride < 1 || a % g || a / g > 16) return hipErrorInvalidValue;
    const int q_heads = a / g, waves = list_waves(simds);
    const bool few = r.max_new * q_heads <= 16;
    // Rows an item: what 16 or 32 columns hold, no more than a sequence has.
    const int m = std::min((few ? 16 : 32) / q_heads, r.max_new);
    const AttnArgs A{r, q, kc, vc, sc, out, part, a, g, m, m * q_heads, (float)(1.4426950408889634 / sqrt((double)D))};
    if (few) {
        hipLaunchKernelGGL((attention_kernel<1, true>), dim3(waves), dim3(64), 0, st, A);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(join_few_kernel, dim3(r.B * g * A.cols), dim3(kJoinThreads), 0, st, A, waves);
        return hipGetLastError();
    }
    const int items = g * (r.rows / m + r.B);
    if (items >= 2 * waves) {
        hipLaunchKernelGGL((attention_kernel<2, false>), dim3(items), dim3(64), 0, st, A);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((attention_kernel<2, true>), dim3(waves), dim3(64), 0, st, A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(join_many_kernel, dim3(waves - 1), dim3(kJoinThreads), 0, st, A, waves);
    return hipGetLastError();
}

}  // namespace kvp
