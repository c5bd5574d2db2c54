// Attention of a call's new rows over the paged bf16 cache: one new token a sequence, a few, or a whole prompt; row i of
// sequence b sits at position len_b + i and sees positions [0, len_b + i], or those of them that lie in its window or below
// `sinks` (WIN).
//
// Columns, items, the list of tiles and the join are attn_rows.h's.  Scores and values on v_mfma_f32_16x16x32_bf16:
//
//   S^T = K Q^T  Row rho of score block tb = 2 s + e is position 32 s + 8 (rho / 4) + 4 e + rho % 4 of the tile, so that lane
//                group grp ends with positions 32 s + 8 grp .. + 7 of its column: the run that a lane of the second product
//                holds, and 16 bytes of a row of V^T.
//   O^T += V^T P^T  The weights, rounded to bf16, go from the score registers into the product as they are; the sum of the
//                weights is taken from the rounded ones, so that their rounding cancels where it is common.
//
// A weight is 0 where its position is hidden, but 0 times a value that is not finite is not.  In tiles that some row of an
// item does not see whole, values that no row sees count as 0, and those that are not finite are taken out of the product
// and put into the rows that see them (as NaN): what a hidden position holds reaches no row.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "attn_rows.h"

namespace kvp {
namespace {

constexpr int kHalfPage = TILE * D;      // values of K, or of V, of one page and head

struct AttnArgs : ListArgs {
    const uint16_t* q;
    const uint16_t* kc;
    const uint16_t* vc;
    float scale_log2;
};

// Bits 15 and 31: whether the bf16 numbers of a word are not finite.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// The halves of a word that are marked in bits 15 and 31, as a mask.
__device__ __forceinline__ uint32_t halves(uint32_t bits) { return (bits >> 15 & 0x10001u) * 0xFFFFu; }

// 16 NB columns of an item, from row t0 of the sequence on.
template <int NB, bool WIN>
struct Columns {
    int lim[NB];             // the last position that the column sees, -1 where there is none
    float m[NB], l[NB];      // running maximum (log2 domain) and sum of the weights
    f32x4 o[NB][8];          // O^T: dimensions 16 db + 4 grp + 0..3 of the column
    int all, last;           // positions up to `all` every row sees (but for its window), past `last` none does
    int low, whole;          // WIN: the first position in the first row's window, and in the last row's

    // Column of block cb: its row, from the item's or wave's first on (past every row where the column
    // is none of the `rows` rows'), and its head.
    static __device__ __forceinline__ int row_of(int cb, int rows, int r) {
        const int c = 16 * cb + (thread_now() & 15);
        return c < rows * r ? c / r : 1 << 30;
    }
    static __device__ __forceinline__ int head_of(int cb, int r) { return (16 * cb + (thread_now() & 15)) % r; }
    static __device__ __forceinline__ int limit(const SeqRows& s, int t0, int rows, int r, int cb) {
        const int t = row_of(cb, rows, r);
        return t < s.act - t0 ? s.len + t0 + t : -1;
    }
    // Queries of the columns: lane (column, grp) holds dimensions 32 ks + 8 grp .. + 7.
    static __device__ __forceinline__ void load_q(const AttnArgs& A, const Item& it, int t0, int rows, u32x4 (&q)[NB][4]) {
        const int grp = (thread_now() >> 4) & 3, r = A.a / A.g;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            const bool real = limit(it.s, t0, rows, r, cb) >= 0;
            const size_t row = it.s.row0 + (real ? t0 + row_of(cb, rows, r) : 0);
            const uint16_t* p = A.q + (row * A.a + it.kvh * r + head_of(cb, r)) * D + 8 * grp;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                q[cb][ks] = u32x4{0, 0, 0, 0};
                if (real) q[cb][ks] = *(const u32x4*)(p + 32 * ks);
            }
        }
    }
    // Begins rows t0 .. t0 + rows - 1 of a sequence (their queries are loaded).
    __device__ __forceinline__ void begin(const AttnArgs& A, const SeqRows& s, int t0, int rows) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            lim[cb] = limit(s, t0, rows, A.a / A.g, cb);
            m[cb] = kNoScore;
            l[cb] = 0.f;
#pragma unroll
            for (int db = 0; db < 8; ++db) o[cb][db] = f32x4{};
        }
        const int n = min(s.act - t0, rows);
        all = n > 0 ? s.len + t0 : -1;
        last = n > 0 ? s.len + t0 + n - 1 : -1;
        if (WIN) {
            low = all - A.window + 1;
            whole = last - A.window + 1;
        }
    }
    // Whether some column does not see all of the tile that begins at p0.
    __device__ __forceinline__ bool edge(const AttnArgs& A, int p0) const {
        return p0 + TILE - 1 > all || (WIN && p0 < whole && p0 + TILE > A.sinks);
    }
    // Whether some column sees some of it.
    __device__ __forceinline__ bool sees(const AttnArgs& A, int p0) const {
        return p0 <= last && (!WIN || p0 + TILE > low || p0 < A.sinks);
    }
    __device__ __forceinline__ bool hidden(const AttnArgs& A, int cb, int p) const {
        return p > lim[cb] || (WIN && p <= lim[cb] - A.window && p >= A.sinks);
    }
    // Whether no column sees position p.
    __device__ __forceinline__ bool unseen(const AttnArgs& A, int p) const { return p > last || (WIN && p < low && p >= A.sinks); }

    // Weights of the tile at p0 from its scores: lane (column, grp) holds positions p0 + 32 s + 8 grp + 4 e + i in block
    // 2 s + e; out: the rows of P, pb.  is_edge: branches around the masks (two copies of this code cost registers).
    __device__ __forceinline__ void softmax(const AttnArgs& A, f32x4 (&sc)[NB][4], bool is_edge, int p0, bf16x8 (&pb)[NB][2]) {
        const int grp = (threadIdx.x >> 4) & 3;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            if (is_edge) {
#pragma unroll
                for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (hidden(A, cb, p0 + 32 * (tb >> 1) + 8 * grp + 4 * (tb & 1) + i)) sc[cb][tb][i] = -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[cb][tb][i]);
            const float mt = pair32_max(pair16_max(mx)) * A.scale_log2;
            if (__any(mt > m[cb] + kLazy)) {
                const float m_new = fmaxf(m[cb], mt);
                const float alpha = __builtin_amdgcn_exp2f(m[cb] - m_new);
                m[cb] = m_new;
                l[cb] *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db) o[cb][db] *= alpha;
            }
            uint32_t pw[8];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[cb][tb][i] = __builtin_amdgcn_exp2f(fmaf(sc[cb][tb][i], A.scale_log2, -m[cb]));
#pragma unroll
            for (int i = 0; i < 8; ++i) pw[i] = pack2bf(sc[cb][i >> 1][2 * (i & 1)], sc[cb][i >> 1][2 * (i & 1) + 1]);
            float lt = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                lt = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[i]),
                                                     __builtin_bit_cast(bf16x2, 0x3F803F80u), lt, false);
            l[cb] += lt;
            pb[cb][0] = as_bf16x8(u32x4{pw[0], pw[1], pw[2], pw[3]});
            pb[cb][1] = as_bf16x8(u32x4{pw[4], pw[5], pw[6], pw[7]});
        }
    }
    // The tile's positions that column cb sees, a bit each.
    __device__ __forceinline__ uint64_t seen(const AttnArgs& A, int cb, int p0) const {
        auto below = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; };
        uint64_t v = below(lim[cb] - p0 + 1);
        if (WIN) v &= ~below(lim[cb] - A.window + 1 - p0) | below(A.sinks - p0);
        return v;
    }
    // Puts the values that are not finite (nf[d]: positions of the tile, a bit each) into the columns that see them.
    __device__ __forceinline__ void spoil(const AttnArgs& A, const uint64_t* nf, int p0) {
        const int grp = (threadIdx.x >> 4) & 3;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            const uint64_t v = seen(A, cb, p0);
            uint32_t bad = 0;
#pragma unroll 1
            for (int k = 0; k < 32; ++k)
                if (nf[16 * (k >> 2) + 4 * grp + (k & 3)] & v) bad |= 1u << k;
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (bad >> k & 1) o[cb][k >> 2][k & 3] = NAN;
        }
    }
    // The end of an item (or of a share inside it): out, or a piece.
    __device__ __forceinline__ void finish(const AttnArgs& A, const Item& it, int t0, int rows, bool to_out, float* piece) {
        const int grp = (thread_now() >> 4) & 3, col = thread_now() & 15, r = A.a / A.g;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            const float lsum = pair32_sum(pair16_sum(l[cb]));
            const int t = row_of(cb, rows, r);
            if (t >= it.s.n - t0) continue;
            if (to_out) {
                const float inv = 1.f / lsum;
                uint16_t* op = A.out + ((size_t)(it.s.row0 + t0 + t) * A.a + it.kvh * r + head_of(cb, r)) * D + 4 * grp;
#pragma unroll
                for (int db = 0; db < 8; ++db) {
                    u32x2 v = {pack2bf(o[cb][db][0] * inv, o[cb][db][1] * inv),
                               pack2bf(o[cb][db][2] * inv, o[cb][db][3] * inv)};
                    if (lim[cb] < 0) v = u32x2{0, 0};      // sees nothing
                    *(u32x2*)(op + 16 * db) = v;
                }
            } else {
                float* pr = piece + (size_t)(16 * cb + col) * PSTRIDE;
#pragma unroll
                for (int db = 0; db < 8; ++db) *(f32x4*)(pr + 16 * db + 4 * grp) = o[cb][db];
                if (grp == 0) {
                    pr[D] = m[cb];
                    pr[D + 1] = lsum;
                }
            }
        }
    }
};

// At most 16 NB columns.  NW 0: a share of the list, one wave.  Else one item, whose tiles NW waves take in turn and
// join in LDS.
template <int NW, int NB, bool WIN>
__global__ __launch_bounds__(NW ? 64 * NW : 64, NW == 8 ? 2 : 1) void rows_few_kernel(AttnArgs A) {
    constexpr bool LIST = NW == 0;
    constexpr int STEP = LIST ? 1 : NW, WAVES = LIST ? 1 : NW;
    __shared__ uint64_t nf[WAVES][D];      // values that are not finite
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    Item it;
    Split sp;
    uint32_t w = 0, left;
    if constexpr (LIST) {
        if (!take_share<true, WIN>(A, &sp, &w, &left, &it)) return;
    } else {
        it.b = blockIdx.x / A.g;
        it.kvh = blockIdx.x % A.g;
        it.s = seq_rows(A.r, it.b);
        if (!it.s.n) return;
        it.c = 0;
        it.t = wave;
        it.template begin<WIN>(A);
        left = max(it.n - wave + NW - 1, 0) / NW;
    }
    Columns<NB, WIN> C;
    u32x4 q[NB][4];
    const int r = A.a / A.g;
    Table<WIN> tab;
    u32x4 k[4][4], v[8][2];      // [score block][32 dimensions], [16-dimension block][32 positions]
    const uint32_t koff = (8 * (col >> 2) + (col & 3)) * D + 8 * grp, voff = col * TILE + 8 * grp;
    auto load_k = [&](size_t at) {
        const uint16_t* p = A.kc + at * kHalfPage;
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) k[tb][ks] = *(const u32x4*)(p + (32 * (tb >> 1) + 4 * (tb & 1)) * D + 32 * ks + koff);
    };
    auto load_v = [&](size_t at) {
        const uint16_t* p = A.vc + at * kHalfPage;
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int s = 0; s < 2; ++s) v[db][s] = *(const u32x4*)(p + 16 * db * TILE + 32 * s + voff);
    };
    bool whole = !LIST || it.t == 0;        // the share has the item from its first tile on
    uint32_t x = LIST ? sp.start(w) : 0;      // the list's tile
    auto begin = [&](const Item& i, uint32_t first) {
        C.begin(A, i.s, i.c * A.m, A.m);
        if (LIST && whole && lane == 0) A.cut[i.b * A.g + i.kvh] = make_int2(w, sp.wave_of(first + i.n - 1) - w + 1);
    };
    C.load_q(A, it, it.c * A.m, A.m, q);
    begin(it, x);
    if (NW < 2 || left) {
        const size_t at = tab.page(A, it);
        load_k(at);
        load_v(at);
    }
    while (NW < 2 || left) {
        // The next tile of the share, perhaps in the next item.
        const bool ends = it.t + STEP >= it.n;
        bool more = left > 1;
        Item nx = it;
        if (more) {
            if (LIST && ends)
                more = next_item<WIN>(A, nx);
            else
                nx.t += STEP;
        }
        const size_t at = more ? tab.page(A, nx) : 0;
        const int p0 = TILE * it.template at<WIN>(A);
        const bool edge = C.edge(A, p0);
        f32x4 sc[NB][4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int cb = 0; cb < NB; ++cb)
                    sc[cb][tb] = mfma16x16x32(as_bf16x8(k[tb][ks]), as_bf16x8(q[cb][ks]), ks ? sc[cb][tb] : f32x4{});
        __builtin_amdgcn_sched_barrier(0);
        // A part of a tile (and the queries) is requested again as soon as it has been multiplied: 16 KB a wave and more
        // are always under way, without a second set of registers.
        if (more) {
            load_k(at);
            if (ends) C.load_q(A, nx, nx.c * A.m, A.m, q);
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pb[NB][2];
        C.softmax(A, sc, edge, p0, pb);
        if (edge) {
            uint32_t any = 0;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = p0 + 32 * s + 8 * grp + 2 * e;
                    const uint32_t mask = (C.unseen(A, p) ? 0u : 0xFFFFu) | (C.unseen(A, p + 1) ? 0u : 0xFFFF0000u);
#pragma unroll
                    for (int db = 0; db < 8; ++db) {
                        v[db][s][e] &= mask;
                        any |= not_finite(v[db][s][e]);
                    }
                }
            if (A.m > 1 && __any(any != 0)) {
                // Rows of an item see different parts of the tile.
#pragma unroll
                for (int db = 0; db < 8; ++db)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        uint32_t bits = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t b = not_finite(v[db][s][e]);
                            bits |= (b >> 15 & 1) << (2 * e) | (b >> 31) << (2 * e + 1);
                            v[db][s][e] &= ~halves(b);
                        }
                        ((uint8_t*)&nf[wave][16 * db + col])[4 * s + grp] = (uint8_t)bits;
                    }
                __builtin_amdgcn_wave_barrier();
                C.spoil(A, nf[wave], p0);
                __builtin_amdgcn_wave_barrier();
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) C.o[cb][db] = mfma16x16x32(as_bf16x8(v[db][s]), pb[cb][s], C.o[cb][db]);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load_v(at);
        if (NW > 1 && !more) break;
        if (ends || !more) {
            C.finish(A, it, it.c * A.m, A.m, whole && ends, A.part + (2 * (size_t)w + (whole ? 1 : 0)) * A.cols * PSTRIDE);
            if (!more) break;
            whole = true;
            begin(nx, x + 1);
        }
        it = nx;
        ++x;
        --left;
    }
    if constexpr (NW > 1) {
        __shared__ float parts[NW][16 * NB][PSTRIDE];
        C.finish(A, it, 0, A.m, false, &parts[wave][0][0]);
        __syncthreads();
        const int cols = min(A.cols, it.s.n * r);
        for (int c = wave; c < cols; c += NW) {
            float M = kNoScore, den = 0.f;
            f32x2 num = {0.f, 0.f};
#pragma unroll
            for (int u = 0; u < NW; ++u) M = fmaxf(M, parts[u][c][D]);
#pragma unroll
            for (int u = 0; u < NW; ++u) {
                const float f = __builtin_amdgcn_exp2f(parts[u][c][D] - M);
                den += f * parts[u][c][D + 1];
                num[0] += f * parts[u][c][2 * lane];
                num[1] += f * parts[u][c][2 * lane + 1];
            }
            const uint32_t o = c / r < it.s.act ? pack2bf(num[0] / den, num[1] / den) : 0u;
            *(uint32_t*)(A.out + ((size_t)(it.s.row0 + c / r) * A.a + it.kvh * r + c % r) * D + 2 * lane) = o;
        }
    }
}

typedef __attribute__((address_space(3))) void lvoid_t;

// Buffer resource of one page and head of K or V at p, the same for the wave (word 3: a valid 32-bit data format).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_buffer(const uint16_t* p) {
    const uint64_t a = (uint64_t)p;
    const uint64_t u = (uint32_t)__builtin_amdgcn_readfirstlane((int)a) |
                       (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32;
    return __builtin_amdgcn_make_buffer_rsrc((void*)u, 0, kHalfPage * 2, 0x00020000);
}

// Eight 16-byte LDS reads and their wait: written by hand, since the compiler would first wait for the loads that go into
// the other stage.  K: the four chunks of two rows' blocks, OFF and OFF + STEP from a0 .. a3; V: four rows' blocks of two
// chunks.
template <int OFF, int STEP>
__device__ __forceinline__ void read_k(uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, u32x4 (&f)[8]) {
    asm volatile("ds_read_b128 %0, %8 offset:%12\n\tds_read_b128 %1, %9 offset:%12\n\t"
                 "ds_read_b128 %2, %10 offset:%12\n\tds_read_b128 %3, %11 offset:%12\n\t"
                 "ds_read_b128 %4, %8 offset:%13\n\tds_read_b128 %5, %9 offset:%13\n\t"
                 "ds_read_b128 %6, %10 offset:%13\n\tds_read_b128 %7, %11 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]),
                   "=&v"(f[7])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "i"(OFF), "i"(OFF + STEP)
                 : "memory");
}
template <int OFF, int STEP>
__device__ __forceinline__ void read_v(uint32_t a0, uint32_t a1, u32x4 (&f)[8]) {
    asm volatile("ds_read_b128 %0, %8 offset:%10\n\tds_read_b128 %1, %9 offset:%10\n\t"
                 "ds_read_b128 %2, %8 offset:%11\n\tds_read_b128 %3, %9 offset:%11\n\t"
                 "ds_read_b128 %4, %8 offset:%12\n\tds_read_b128 %5, %9 offset:%12\n\t"
                 "ds_read_b128 %6, %8 offset:%13\n\tds_read_b128 %7, %9 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]),
                   "=&v"(f[7])
                 : "v"(a0), "v"(a1), "i"(OFF), "i"(OFF + STEP), "i"(OFF + 2 * STEP), "i"(OFF + 3 * STEP)
                 : "memory");
}

// Workgroup: an item of 4 mw rows, wave v's 16 NB columns are its rows v mw .. (v + 1) mw - 1.  The tiles go from memory to
// LDS directly, two stages of 32 KB, one barrier a tile: it ends the loads of the tile that comes and the reads of the one
// before it, whose stage is then loaded again.  Two workgroups a CU run in each other's waits.
// LIST: a share of the list; else one item, counted from a sequence's last.
template <bool LIST, int NB, bool WIN>
__global__ __launch_bounds__(256, 2) void rows_many_kernel(AttnArgs A) {
    // K: chunk c (16 bytes, 8 dimensions) of row R at place c ^ key(R) of its 16, key of the bits that differ among the 16 rows
    // of a fragment; V^T: chunk c (8 positions) of row d at place c ^ (d / 2 % 8) of its 8: the 16 lanes of a group fall on all
    // banks.
    __shared__ u32x4 kl[2][TILE * 16], vl[2][D * 8];
    __shared__ uint64_t nf[D];             // values that are not finite
    auto key = [](int R) { return (R & 3) | ((R >> 3) & 3) << 2; };
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Item it;
    uint32_t w = 0, left;
    if constexpr (LIST) {
        Split sp;
        if (!take_share<false, WIN>(A, &sp, &w, &left, &it)) {
            if (tid == 0) A.cut_many[blockIdx.x].np = 0;
            return;
        }
        // The item that the share begins and does not end: that of its last tile.
        if (tid < 64) {
            CutItem cut{};
            if (w + 1 < sp.W) {
                const uint32_t xe = sp.start(w + 1) - 1;
                Lanes<false, WIN> L;
                list_tiles<false, WIN>(A, L);
                const Item e = find_tile<false, WIN>(A, L, xe);
                if (e.t + 1 < e.n && xe - e.t >= sp.start(w)) {
                    cut.np = sp.wave_of(xe - e.t + e.n - 1) - w + 1;
                    cut.row = e.s.row0 + e.c * A.m;
                    cut.n = e.s.n - e.c * A.m;
                    cut.act = e.s.act - e.c * A.m;
                    cut.head = e.kvh * (A.a / A.g);
                }
            }
            if (tid == 0) A.cut_many[w] = cut;
        }
    } else {
        // The last block of every sequence first, as the longest, and so on; K/V heads change fastest: with
        // 8 of them each XCD reads one of them only.
        const int x = blockIdx.x / A.g;
        it.kvh = blockIdx.x % A.g;
        it.b = x % A.r.B;
        it.c = gridDim.x / (A.r.B * A.g) - 1 - x / A.r.B;
        it.s = seq_rows(A.r, it.b);
        if (it.c >= blocks_of(it.s, A.m)) return;
        it.t = 0;
        it.template begin<WIN>(A);
        left = it.n;
    }
    const int r = A.a / A.g, wcols = A.mw * r;
    Columns<NB, WIN> C;
    u32x4 q[NB][4];
    Table<WIN> tab;
    auto issue = [&](const Item& i, int stg) {
        const size_t at = tab.page(A, i);
        const __amdgpu_buffer_rsrc_t kr = page_buffer(A.kc + at * kHalfPage), vr = page_buffer(A.vc + at * kHalfPage);
        // The lane's 16 bytes of each of this wave's four KB of K (rows 16 wave + 4 i + lane / 16) and of V^T (rows
        // 32 wave + 8 i + lane / 8).
        const int now = thread_now() & 63;
        const uint32_t ksrc = (now >> 4) * (2 * D) + 16 * ((now & 15) ^ ((now >> 4) | ((2 * wave) & 3) << 2));
        const uint32_t vsrc = (now >> 3) * (2 * TILE) + 16 * ((now & 7) ^ (now >> 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lvoid_t*)&kl[stg][256 * wave + 64 * i], 16, i < 2 ? ksrc : ksrc ^ 64u,
                                                     4096 * wave + 1024 * i, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lvoid_t*)&vl[stg][256 * wave + 64 * i], 16, i & 1 ? vsrc ^ 64u : vsrc,
                                                     4096 * wave + 1024 * i, 0, 0);
        }
    };
    bool whole = it.t == 0;
    int t0 = it.c * A.m + wave * A.mw;        // the wave's first row
    issue(it, 0);
    C.load_q(A, it, t0, A.mw, q);
    C.begin(A, it.s, t0, A.mw);
    for (int stg = 0;; stg ^= 1) {
        const bool ends = it.t + 1 == it.n;
        bool more = left > 1;
        Item nx = it;
        if (more) {
            if (LIST && ends)
                more = next_item<WIN>(A, nx);
            else
                ++nx.t;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wave's part of the tile is in LDS
        __syncthreads();
        const int p0 = TILE * it.template at<WIN>(A);
        // Values that not all of the item's rows see.
        bool spoilt = false;
        {
            Columns<1, WIN> B;       // the item's rows
            const int n = min(it.s.act - it.c * A.m, A.m);
            B.all = n > 0 ? it.s.len + it.c * A.m : -1;
            B.last = B.all + n - 1;
            if (n <= 0) B.last = -1;
            if (WIN) B.low = B.all - A.window + 1, B.whole = B.last - A.window + 1;
            if (B.edge(A, p0)) {
                bool bad = false;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = thread_now() + 256 * j, d = i >> 3, c = (i & 7) ^ ((d >> 1) & 7);
                    u32x4 x = vl[stg][i];
                    uint32_t bits = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int p = p0 + 8 * c + 2 * e;
                        x[e] &= (B.unseen(A, p) ? 0u : 0xFFFFu) | (B.unseen(A, p + 1) ? 0u : 0xFFFF0000u);
                        const uint32_t b = not_finite(x[e]);
                        bits |= (b >> 15 & 1) << (2 * e) | (b >> 31) << (2 * e + 1);
                        x[e] &= ~halves(b);
                    }
                    vl[stg][i] = x;
                    ((uint8_t*)&nf[d])[c] = (uint8_t)bits;
                    bad |= bits != 0;
                }
                spoilt = __syncthreads_or(bad);
            }
        }
        if (more) issue(nx, stg ^ 1);
        if (C.sees(A, p0)) {
            const bool edge = C.edge(A, p0);
            if (spoilt) C.spoil(A, nf, p0);
            f32x4 sc[NB][4];
            const int now = thread_now(), col = now & 15, grp = (now >> 4) & 3;
            // The lane's rows of the four score blocks have one key; their chunks 4 ks + grp.
            const int krow = 8 * (col >> 2) + (col & 3), kk = key(krow);
            const uint32_t kb = (uint32_t)(uintptr_t)&kl[stg][krow * 16];
            const uint32_t k0 = kb + 16 * (grp ^ kk), k1 = kb + 16 * ((4 + grp) ^ kk), k2 = kb + 16 * ((8 + grp) ^ kk),
                           k3 = kb + 16 * ((12 + grp) ^ kk);
            auto scores = [&](auto tb_t) __attribute__((always_inline)) {
                constexpr int s = decltype(tb_t)::value;      // blocks 2 s and 2 s + 1: rows 32 s, 32 s + 4 further
                u32x4 f[8];
                read_k<s * 32 * 2 * D, 4 * 2 * D>(k0, k1, k2, k3, f);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int cb = 0; cb < NB; ++cb)
                            sc[cb][2 * s + e] = mfma16x16x32(as_bf16x8(f[4 * e + ks]), as_bf16x8(q[cb][ks]),
                                                             ks ? sc[cb][2 * s + e] : f32x4{});
            };
            __builtin_amdgcn_s_setprio(1);
            scores(std::integral_constant<int, 0>{});
            scores(std::integral_constant<int, 1>{});
            __builtin_amdgcn_s_setprio(0);
            bf16x8 pb[NB][2];
            C.softmax(A, sc, edge, p0, pb);
            const uint32_t vb = (uint32_t)(uintptr_t)&vl[stg][col * 8];
            const uint32_t v0 = vb + 16 * (grp ^ ((col >> 1) & 7)), v1 = v0 ^ 64u;
            auto vals = [&](auto d0_t) __attribute__((always_inline)) {
                constexpr int d0 = decltype(d0_t)::value;
                u32x4 f[8];
                read_v<d0 * 16 * 2 * TILE, 16 * 2 * TILE>(v0, v1, f);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int cb = 0; cb < NB; ++cb)
                            C.o[cb][d0 + i] = mfma16x16x32(as_bf16x8(f[2 * i + s]), pb[cb][s], C.o[cb][d0 + i]);
            };
            __builtin_amdgcn_s_setprio(1);
            vals(std::integral_constant<int, 0>{});
            vals(std::integral_constant<int, 4>{});
            __builtin_amdgcn_s_setprio(0);
        }
        if (ends || !more) {
            float* piece = A.part + ((2 * (size_t)w + (whole ? 1 : 0)) * A.cols + wave * wcols) * PSTRIDE;
            C.finish(A, it, t0, A.mw, whole && ends, piece);
            if (!more) break;
            whole = true;
            t0 = nx.c * A.m + wave * A.mw;
            C.load_q(A, nx, t0, A.mw, q);
            C.begin(A, nx.s, t0, A.mw);
        }
        it = nx;
        --left;
    }
}

// Shares of the list: one wave a SIMD of few columns, as many workgroups as a CU holds of many.
int few_shares(int simds) { return std::min(simds, kMaxDecodeSplits); }
int many_shares(int simds) { return std::max(1, 2 * simds / 4); }

constexpr int kFewCols = 32;      // up to here a wave takes all columns of an item
template <int NB, bool WIN>
void launch_few(int nw, int grid, const AttnArgs& A, hipStream_t st) {
    constexpr int MOST = NB == 1 ? 8 : 4;       // waves of a workgroup that have the registers for it
    if (nw == 0) hipLaunchKernelGGL((rows_few_kernel<0, NB, WIN>), dim3(grid), dim3(64), 0, st, A);
    else if (nw == 1) hipLaunchKernelGGL((rows_few_kernel<1, NB, WIN>), dim3(grid), dim3(64), 0, st, A);
    else if (nw == 2) hipLaunchKernelGGL((rows_few_kernel<2, NB, WIN>), dim3(grid), dim3(128), 0, st, A);
    else hipLaunchKernelGGL((rows_few_kernel<MOST, NB, WIN>), dim3(grid), dim3(64 * MOST), 0, st, A);
}
template <int NB, bool WIN>
void launch_many(bool list, int grid, const AttnArgs& A, hipStream_t st) {
    if (list) hipLaunchKernelGGL((rows_many_kernel<true, NB, WIN>), dim3(grid), dim3(256), 0, st, A);
    else hipLaunchKernelGGL((rows_many_kernel<false, NB, WIN>), dim3(grid), dim3(256), 0, st, A);
}

// Waves that take an item of few columns where a launch without a list and a join is the faster one, else 0.  tiles: of
// the longest item.
int few_waves(int64_t items, int64_t tiles, int simds) {
    if (tiles <= 2) return 1;
    if (tiles > std::min<int64_t>(32, 14 + items / 4)) return 0;
    return items <= simds / 4 ? 8 : items <= simds / 2 ? 2 : 1;
}

template <bool WIN>
hipError_t launch(AttnArgs& A, int simds, hipStream_t st) {
    const NewRows& r = A.r;
    const int heads = A.a / A.g;
    // The most tiles that an item of m rows can have.
    auto most = [&](int m) -> int64_t {
        const int64_t n = r.max_pos / TILE + 1;
        if (!WIN) return n;
        return std::min<int64_t>(n, ((int64_t)A.window + m + TILE - 2) / TILE + 1 + (A.sinks + TILE - 1) / TILE);
    };
    // The list counts tiles in 31 bits; where it might not, items run one by one.
    auto listed = [&](int64_t items, int m) { return items * most(m) <= INT32_MAX; };
    hipError_t e;
    if (r.max_new * heads <= kFewCols) {
        A.m = r.max_new;
        A.cols = A.m * heads;
        const int items = r.B * A.g, nw = listed(items, A.m) ? few_waves(items, most(A.m), simds) : 1;
        if (nw) {
            if (A.cols <= 16) launch_few<1, WIN>(nw, items, A, st);
            else launch_few<2, WIN>(nw, items, A, st);
            return hipGetLastError();
        }
        const int shares = few_shares(simds);
        A.cut = (int2*)(A.part + (size_t)2 * shares * A.cols * PSTRIDE);
        if (A.cols <= 16) launch_few<1, WIN>(0, shares, A, st);
        else launch_few<2, WIN>(0, shares, A, st);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        // Few pieces an item, a wave a column; many, four waves.
        if (shares <= 32 * items)
            hipLaunchKernelGGL(join_short_kernel, dim3((items * A.cols + kJoinWaves - 1) / kJoinWaves), dim3(kJoinThreads), 0, st, A);
        else
            hipLaunchKernelGGL(join_few_kernel, dim3(items * A.cols), dim3(kJoinThreads), 0, st, A);
        return hipGetLastError();
    }
    // Rows of a wave: what its 16 (where they hold a quarter of the longest sequence's rows) or 32 columns hold, and no
    // more than that quarter.
    const int nb = 4 * (16 / heads) >= r.max_new ? 1 : 2;
    A.mw = std::min(16 * nb / heads, (r.max_new + 3) / 4);
    A.m = 4 * A.mw;
    A.cols = A.m * heads;
    const int shares = many_shares(simds);
    const int64_t items = (int64_t)A.g * (r.rows / A.m + r.B), grid = (int64_t)A.g * r.B * ((r.max_new + A.m - 1) / A.m);
    // Items one by one or the list, in us.  One by one: the tiles of the longest one after the other, a part of all
    // work, and blocks that are none (the grid has as many for every sequence as the longest may have).  The list: all
    // work shared evenly, a second launch, and the pieces' way to memory and back.  Of the tiles some 0.6 of the most
    // that there may be.
    const double n = most(A.m), T = 0.6 * items * n;
    const double one = 6 + 1.65 * n + T / 512 + grid / 2000.,
                 list = 12 + T / 256 + (std::min<double>(T, shares) + items) * A.cols * (PSTRIDE * sizeof(float)) / 2.3e6;
    const bool fits = grid < 1 << 24;       // 2^32 threads
    if ((one < list && fits) || !listed(items, A.m)) {
        if (!fits) return hipErrorInvalidValue;
        nb == 1 ? launch_many<1, WIN>(false, grid, A, st) : launch_many<2, WIN>(false, grid, A, st);
        return hipGetLastError();
    }
    A.cut_many = (CutItem*)(A.part + (size_t)2 * shares * A.cols * PSTRIDE);
    nb == 1 ? launch_many<1, WIN>(true, shares, A, st) : launch_many<2, WIN>(true, shares, A, st);
    if ((e = hipGetLastError()) != hipSuccess || shares == 1) return e;
    const dim3 join(shares - 1, (A.cols + kJoinCols - 1) / kJoinCols);
    if (4 * items <= shares)
        hipLaunchKernelGGL(join_long_kernel, join, dim3(kJoinThreads), 0, st, A);
    else
        hipLaunchKernelGGL(join_many_kernel, join, dim3(kJoinThreads), 0, st, A);
    return hipGetLastError();
}

}  // namespace

// Pieces, then what the join reads.
size_t attention_rows_bytes(int B, int g, int simds) {
    const size_t pieces = (size_t)2 * PSTRIDE * sizeof(float) * std::max(kFewCols * few_shares(simds), 128 * many_shares(simds));
    return pieces + std::max((size_t)B * g * sizeof(int2), (size_t)many_shares(simds) * sizeof(CutItem));
}

hipError_t attention_rows(const NewRows& r, int a, int g, int window, int sinks, const uint16_t* q, const uint16_t* kc,
                          const uint16_t* vc, uint16_t* out, void* ws, int simds, hipStream_t st) {
    if (r.B < 1 || r.rows < 1 || r.n_pages < 1 || r.stride < 1 || a % g || a / g > 16 || window < 0 || sinks < 0)
        return hipErrorInvalidValue;
    AttnArgs A{{r, out, (float*)ws, a, g}, q, kc, vc, (float)(1.4426950408889634 / sqrt((double)D))};
    // A window that hides nothing from any row is none.
    if (window == 0 || (int64_t)window + sinks > r.max_pos) return launch<false>(A, simds, st);
    A.window = window;
    A.sinks = sinks;
    return launch<true>(A, simds, st);
}

}  // namespace kvp
