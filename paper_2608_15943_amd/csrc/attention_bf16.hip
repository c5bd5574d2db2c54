// Attention of a call's new rows over the paged bf16 cache: one new token a sequence, a few, or a whole prompt; row i of
// sequence b sits at position len_b + i and sees positions [0, len_b + i], or those of them that lie in its window or below
// `sinks` (WIN).
//
// Columns, items, the list of tiles of few columns and its join are attn_rows.h's; items of more columns run whole or in
// parts (take_part).  Scores and values on v_mfma_f32_16x16x32_bf16:
//
//   S^T = K Q^T  Row rho of score block tb = 2 s + e is position 32 s + 8 (rho / 4) + 4 e + rho % 4 of the tile, so that lane
//                group grp ends with positions 32 s + 8 grp .. + 7 of its column: the run that a lane of the second product
//                holds, and 16 bytes of a row of V^T.
//   O^T += V^T P^T  The weights, rounded to bf16, go from the score registers into the product as they are; the sum of the
//                weights is taken from the rounded ones, so that their rounding cancels where it is common.
//
// A weight is 0 where its position is hidden, but 0 times a value that is not finite is not.  In tiles that some row of an
// item does not see whole, values that are not finite are taken out of the product and put, as NaN, into the rows that see
// them: what a hidden position holds reaches no row.
#include <math.h>

#include <algorithm>

#include "attn_rows.h"
#include "part_length.h"

namespace kvp {
namespace {

constexpr int kHalfPage = TILE * D;      // values of K, or of V, of one page and head

struct AttnArgs : ListArgs {
    const uint16_t* q;
    const uint16_t* kc;
    const uint16_t* vc;
    float scale_log2;
    // Of many columns: tiles and parts of an item at most; or the parts of all items together.
    int longest, parts, jobs;
};

// Bits 15 and 31: whether the bf16 numbers of a word are not finite.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// The halves of a word that are marked in bits 15 and 31, as a mask.
__device__ __forceinline__ uint32_t halves(uint32_t bits) { return (bits >> 15 & 0x10001u) * 0xFFFFu; }

// What rows t0 .. t0 + rows - 1 of a sequence see together.
template <bool WIN>
struct Span {
    int all, last;           // positions up to `all` every row sees (but for its window), past `last` none does
    int low, whole;          // WIN: the first position in the first row's window, and in the last row's
    Span() = default;
    __device__ __forceinline__ Span(const ListArgs& A, const SeqRows& s, int t0, int rows) {
        const int n = min(s.act - t0, rows);
        all = n > 0 ? s.len + t0 : -1;
        last = n > 0 ? s.len + t0 + n - 1 : -1;
        low = WIN ? all - A.window + 1 : 0;
        whole = WIN ? last - A.window + 1 : 0;
    }
    // Whether some row does not see all of the tile that begins at p0.
    __device__ __forceinline__ bool edge(const ListArgs& A, int p0) const {
        return p0 + TILE - 1 > all || (WIN && p0 < whole && p0 + TILE > A.sinks);
    }
    // Whether some row sees some of it.
    __device__ __forceinline__ bool sees(const ListArgs& A, int p0) const {
        return p0 <= last && (!WIN || p0 + TILE > low || p0 < A.sinks);
    }
    // Whether no row sees position p.
    __device__ __forceinline__ bool unseen(const ListArgs& A, int p) const {
        return p > last || (WIN && p < low && p >= A.sinks);
    }
};

// 16 NB columns of an item, from row t0 of the sequence on.
template <int NB, bool WIN>
struct Columns : Span<WIN> {
    int lim[NB];             // the last position that the column sees, -1 where there is none
    float m[NB], l[NB];      // running maximum (log2 domain) and sum of the weights
    f32x4 o[NB][8];          // O^T: dimensions 16 db + 4 grp + 0..3 of the column

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
        *(Span<WIN>*)this = Span<WIN>(A, s, t0, rows);
    }
    // Hides what a column does not see of the tile at p0 in its scores (lane (column, grp) holds positions p0 + 32 s + 8 grp +
    // 4 e + i in block 2 s + e) and moves the running maxima.
    __device__ __forceinline__ void maxima(const AttnArgs& A, f32x4 (&sc)[NB][4], bool is_edge, int p0) {
        const int grp = (threadIdx.x >> 4) & 3;
        if (is_edge) {
            const int at = p0 + 8 * grp;          // the lane's first position; the others are constants further
#pragma unroll
            for (int cb = 0; cb < NB; ++cb) {
                const int hi = lim[cb] - at, lo = hi - A.window, sk = A.sinks - at;
#pragma unroll
                for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int off = 32 * (tb >> 1) + 4 * (tb & 1) + i;
                        if (off > hi || (WIN && off <= lo && off >= sk)) sc[cb][tb][i] = -INFINITY;
                    }
            }
        }
        // The lanes of a column look at their own scores first: the maxima move rarely.
        float mx[NB];
        bool moves = false;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            mx[cb] = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx[cb] = fmaxf(mx[cb], sc[cb][tb][i]);
            moves |= mx[cb] * A.scale_log2 > m[cb] + kLazy;
        }
        if (__any(moves)) {
#pragma unroll
            for (int cb = 0; cb < NB; ++cb) {
                const float mt = pair32_max(pair16_max(mx[cb])) * A.scale_log2;
                if (mt > m[cb] + kLazy) {
                    const float alpha = __builtin_amdgcn_exp2f(m[cb] - mt);
                    m[cb] = mt;
                    l[cb] *= alpha;
#pragma unroll
                    for (int db = 0; db < 8; ++db) o[cb][db] *= alpha;
                }
            }
        }
    }
    // The tile's weights, the rows of P, and their sums.
    __device__ __forceinline__ void weights(const AttnArgs& A, const f32x4 (&sc)[NB][4], bf16x8 (&pb)[NB][2]) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            uint32_t pw[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                pw[i] = pack2bf(__builtin_amdgcn_exp2f(fmaf(sc[cb][i >> 1][2 * (i & 1)], A.scale_log2, -m[cb])),
                                __builtin_amdgcn_exp2f(fmaf(sc[cb][i >> 1][2 * (i & 1) + 1], A.scale_log2, -m[cb])));
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

// At most 16 NB columns.  NW 0: a share of the list, or (A.parts) a part of an item, one wave.  Else one item, whose tiles NW waves take in turn and
// join in LDS.
//
// Bound by memory: K and V are read once, straight into registers, 32 KB a tile and one wave a SIMD, which has 16 to 32 KB
// requested at any time; a tile takes 5.5 us of the device's rate and some 1 us of vector and matrix work beside it.  64
// sequences behind 16384 positions (32 heads on 8; 4.3 GB) 704 us, 6.1 TB/s, what a bare read reaches; 64 behind 3000-40000 in
// windows of 4096 (1.07 GB) 195 us, 5.5 TB/s; 16 x 4 rows behind 1500-8000 (312 MB) 63 us, 4.9 TB/s: 9 or 10 tiles a wave, the
// first behind the list, a length, a page number and a page, one after the other.  The join takes 4 to 5 us more.
template <int NW, int NB, bool WIN>
__global__ __launch_bounds__(NW ? 64 * NW : 64, 1) void rows_few_kernel(AttnArgs A) {
    constexpr bool LIST = NW == 0;
    constexpr int STEP = LIST ? 1 : NW, WAVES = LIST ? 1 : NW;
    __shared__ uint64_t nf[WAVES][D];      // values that are not finite
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    Item it;
    Split sp;
    uint32_t w = 0, left;
    int pieces = 0;                        // LIST: of the item, 0: of even shares
    if constexpr (LIST) {
        if (A.parts) {
            const int item = blockIdx.x % (A.r.B * A.g), part = blockIdx.x / (A.r.B * A.g);
            it.b = item / A.g;
            it.kvh = item % A.g;
            it.s = seq_rows(A.r, it.b);
            if (!it.s.n) return;
            it.c = 0;
            it.template begin<WIN>(A);
            pieces = min(it.n, A.parts);
            if (part >= pieces) return;
            it.t = (int)((int64_t)it.n * part / pieces);
            left = (int)((int64_t)it.n * (part + 1) / pieces) - it.t;
            w = item * A.parts + part;
        } else if (!take_share<true, WIN>(A, &sp, &w, &left, &it)) {
            return;
        }
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
    uint32_t x = LIST && !pieces ? sp.start(w) : 0;      // the list's tile
    auto begin = [&](const Item& i, uint32_t first) {
        C.begin(A, i.s, i.c * A.m, A.m);
        if (LIST && whole && lane == 0)
            A.cut[i.b * A.g + i.kvh] = make_int2(w, pieces ? pieces : (int)(sp.wave_of(first + i.n - 1) - w) + 1);
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
        C.maxima(A, sc, edge, p0);
        C.weights(A, sc, pb);
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

typedef int i32x4 __attribute__((ext_vector_type(4)));
// Buffer resource of one page and head of K or V at p, the same for the wave (word 3: a valid 32-bit data format).
__device__ __forceinline__ i32x4 page_buffer(const uint16_t* p) {
    const uint64_t a = (uint64_t)p;
    return i32x4{__builtin_amdgcn_readfirstlane((int)a), __builtin_amdgcn_readfirstlane((int)(a >> 32) & 0xFFFF), kHalfPage * 2,
                 0x00020000};
}
// Four KB of a page into LDS at `lds` (both the same for the wave), 16 bytes a lane and KB: the lane's bytes lie at v0 of
// the first KB, at v1, v2 and v3 of the others.  In assembly, so that the compiler, which cannot tell the stages of a tile
// apart, does not wait for these loads before every read of LDS; they write nothing but LDS, m0 is as it was, and the caller
// waits.
__device__ __forceinline__ void load_4kb(i32x4 page, uint32_t lds, uint32_t at, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\t"
                 "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %5, %9, %10 offen lds\n\t"
                 "s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %6, %9, %11 offen lds\n\t"
                 "s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %7, %9, %12 offen lds\n\t"
                 "s_mov_b32 m0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %8, %9, %13 offen lds\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "s"(lds), "s"(lds + 1 * 1024), "s"(lds + 2 * 1024), "s"(lds + 3 * 1024), "v"(v0), "v"(v1), "v"(v2), "v"(v3), "s"(page),
                   "s"(at), "s"(at + 1 * 1024), "s"(at + 2 * 1024), "s"(at + 3 * 1024)
                 : "memory");
}

// 16 fragments of NB products each, their LDS reads four fragments ahead of them.
template <int SYNC, int NB>
__device__ __forceinline__ void reads_ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, 4, SYNC);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, NB, SYNC);
        if (i < 12) __builtin_amdgcn_sched_group_barrier(0x100, 1, SYNC);
    }
}

// A bound of the tiles of every block of a sequence (without a window that of its last row).
template <bool WIN>
__device__ __forceinline__ int most_tiles(const ListArgs& A, const SeqRows& s) {
    const int n = s.act ? (s.len + s.act - 1) / TILE + 1 : 1;
    return WIN ? min(n, (A.window + A.m + TILE - 2) / TILE + 1 + sink_tiles(A)) : n;
}
// An item, or a part of it, as a workgroup takes it.
struct Part {
    Item it;
    int part, parts;
    int slot, step;          // of its first piece, from one to the next
};
// The item, or part, of workgroup x; join: the item whose parts workgroup x joins.  False: there is none.
//
// By length (A.jobs 0): a grid of A.parts x the longest sequence's blocks x B x g, parts of A.longest tiles at most.  The last
// block of every sequence first, as the longest, and so on; the blocks' last parts before all others.
// By count: A.jobs parts at most, so long that they are no more; sequence by sequence, the first parts of its items first.
// Either way parts that run together read the same positions at about the same time, and share them in L2.  K/V heads
// change fastest: with 8 of them each XCD reads one of them only.
template <bool WIN>
__device__ __forceinline__ bool take_part(const AttnArgs& A, int x, bool join, Part* p) {
    Item& it = p->it;
    int longest = A.longest;
    if (!A.jobs) {
        const int blocks = (A.r.max_new + A.m - 1) / A.m;
        it.kvh = x % A.g;
        x /= A.g;
        it.b = x % A.r.B;
        x /= A.r.B;
        it.c = blocks - 1 - x % blocks;
        p->part = join ? 0 : A.parts - 1 - x / blocks;
        it.s = seq_rows(A.r, it.b);
        if (it.c >= blocks_of(it.s, A.m)) return false;
        // The sequences before it have row0 / m + b blocks at most.
        p->slot = ((it.s.row0 / A.m + it.b + it.c) * A.g + it.kvh) * A.parts;
        p->step = 1;
    } else {
        const int lane = threadIdx.x & 63;
        // Items, and tiles if all blocks had as many as their sequence's longest.  Sums alone, so that every workgroup finds the
        // same length.
        SeqRows s{0, 0, 0, 0};
        int items = 0;
        float n_lane = 0.f;
        uint64_t t_lane = 0;
        for (int b0 = 0; b0 < A.r.B; b0 += 64) {
            items = 0;
            if (b0 + lane < A.r.B) {
                s = seq_rows(A.r, b0 + lane);
                items = blocks_of(s, A.m) * A.g;
                n_lane += (float)items;
                t_lane += (uint64_t)items * most_tiles<WIN>(A, s);
            }
        }
        longest = __builtin_amdgcn_readfirstlane(part_length(A.jobs, wave_sum(n_lane), wave_sum((float)t_lane)));
        int item0 = 0, job0 = 0, n = 0;
        for (int b0 = 0;; b0 += 64) {
            if (b0 >= A.r.B) return false;
            if (A.r.B > 64) {
                items = 0;
                if (b0 + lane < A.r.B) {
                    s = seq_rows(A.r, b0 + lane);
                    items = blocks_of(s, A.m) * A.g;
                }
            }
            const int tiles = items ? most_tiles<WIN>(A, s) : 0, k = parts_of(tiles, longest), jobs = items * k;
            int ie = 0, je = 0;            // before this lane's sequence
            if (A.r.B <= 8) {
                // The sequence of the longest parts first: a few sequences end with short ones (3 chunks 118 us, in their order
                // 127; 6 of 13-900 rows 104, 113).  Many mix the long contexts of few rows, bound by memory, with the rest in
                // any order, and are slower sorted (8: 132 and 134 us; 16: 123 and 109; 32: 127 and 114).
                const int each = k ? (tiles + k - 1) / k : 0;
                for (int i = 0; i < A.r.B; ++i) {
                    const int e = __builtin_amdgcn_readlane(each, i), u = __builtin_amdgcn_readlane(items, i),
                              v = __builtin_amdgcn_readlane(jobs, i);
                    if (e > each || (e == each && i < lane)) ie += u, je += v;
                }
            } else {
                ie = items, je = jobs;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const int u = __shfl_up(ie, off), v = __shfl_up(je, off);
                    if (lane >= off) ie += u, je += v;
                }
                ie -= items, je -= jobs;
            }
            const int at = x - (join ? item0 + ie : job0 + je);
            const uint64_t here = __ballot(at >= 0 && at < (join ? items : jobs));
            if (here) {
                const int w = __builtin_ctzll(here);
                it.b = b0 + w;
                it.s = {__builtin_amdgcn_readlane(s.row0, w), __builtin_amdgcn_readlane(s.n, w), __builtin_amdgcn_readlane(s.len, w),
                        __builtin_amdgcn_readlane(s.act, w)};
                n = __builtin_amdgcn_readlane(items, w);
                item0 += __builtin_amdgcn_readlane(ie, w);
                job0 += __builtin_amdgcn_readlane(je, w);
                break;
            }
            item0 += __builtin_amdgcn_readlane(ie + items, 63);
            job0 += __builtin_amdgcn_readlane(je + jobs, 63);
        }
        x -= join ? item0 : job0;
        p->part = x / n;
        x %= n;
        it.kvh = x % A.g;
        it.c = n / A.g - 1 - x / A.g;
        p->slot = job0 + x;
        p->step = n;
    }
    it.template begin<WIN>(A);
    p->parts = parts_of(it.n, longest);
    return p->part < p->parts;
}

// Workgroup: a part of an item of 4 mw rows, wave v's 16 NB columns are its rows v mw .. (v + 1) mw - 1.  The tiles go from
// memory to LDS directly, two stages of 32 KB, one barrier a tile: it ends the loads of the tile that comes and the reads of
// the one before it, whose stage is then loaded again.  Two workgroups a CU run in each other's waits.
//
// Bound by LDS and the matrix and vector units together.  A fragment of K or V that is read from LDS serves NB products: of 16
// columns a wave the reads take longer than the products (8192 rows, 64 heads on 8: 1220 us), of 32 about as long (980), of 48
// less (912 us, 1207 TFLOP/s; a large product of the library 1310-1400), with 242 of 256 registers; of 64 the accumulators
// leave the first half of the registers (slower).  The reads of fragments run four ahead of the products.  The exponentials of
// a tile take about half the products' time and run beside the other workgroup's.
// Other ways, both slower: K a tile ahead of the softmax, and loads by the compiler's builtin, which waits for them before
// reads of LDS (prompts of 4 x 4096 and 8192 rows 1 %, chunks and windows 3 %).
template <int NB, bool WIN>
__global__ __launch_bounds__(256, 2) void rows_many_kernel(AttnArgs A) {
    // K: chunk c (16 bytes, 8 dimensions) of row R at place c ^ key(R) of its 16, key of the bits that differ among the 16 rows
    // of a fragment; V^T: chunk c (8 positions) of row d at place c ^ (d / 2 % 8) of its 8: the 16 lanes of a group fall on all
    // banks.
    __shared__ u32x4 kl[2][TILE * 16], vl[2][D * 8];
    __shared__ uint64_t nf[D];             // values that are not finite
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Part P;
    if (!take_part<WIN>(A, blockIdx.x, false, &P)) return;
    Item& it = P.it;
    const int end = (int)((int64_t)it.n * (P.part + 1) / P.parts);
    it.t = (int)((int64_t)it.n * P.part / P.parts);
    const int r = A.a / A.g, wcols = A.mw * r;
    Columns<NB, WIN> C;
    u32x4 q[NB][4];
    Table<WIN> tab;
    // The lane's 16 bytes of each of this wave's four KB of K (rows 16 wave + 4 i + lane / 16) and of V^T (rows
    // 32 wave + 8 i + lane / 8).
    auto issue = [&](size_t at, int stg) __attribute__((always_inline)) {
        const int now = thread_now() & 63;
        const uint32_t ksrc = (now >> 4) * (2 * D) + 16 * ((now & 15) ^ ((now >> 4) | ((2 * wave) & 3) << 2));
        const uint32_t vsrc = (now >> 3) * (2 * TILE) + 16 * ((now & 7) ^ (now >> 4));
        const uint32_t kd = (uint32_t)(uintptr_t)&kl[stg][256 * wave], vd = (uint32_t)(uintptr_t)&vl[stg][256 * wave];
        load_4kb(page_buffer(A.kc + at * kHalfPage), __builtin_amdgcn_readfirstlane(kd), 4096 * wave, ksrc, ksrc, ksrc ^ 64u, ksrc ^ 64u);
        load_4kb(page_buffer(A.vc + at * kHalfPage), __builtin_amdgcn_readfirstlane(vd), 4096 * wave, vsrc, vsrc ^ 64u, vsrc, vsrc ^ 64u);
    };
    // Scores of a K stage: the lane's rows of the four score blocks have one key; their chunks 4 ks + grp.
    const int col = tid & 15, grp = (tid >> 4) & 3;
    const int krow = 8 * (col >> 2) + (col & 3), kk = (krow & 3) | ((krow >> 3) & 3) << 2;
    auto scores = [&](const u32x4* kl, f32x4 (&z)[NB][4]) __attribute__((always_inline)) {
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const bf16x8 f = as_bf16x8(kl[(krow + 32 * (tb >> 1) + 4 * (tb & 1)) * 16 + ((4 * ks + grp) ^ kk)]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) z[cb][tb] = mfma16x16x32(f, as_bf16x8(q[cb][ks]), ks ? z[cb][tb] : f32x4{});
            }
        reads_ahead<0, NB>();
    };
    auto values = [&](const u32x4* vl, const bf16x8 (&pb)[NB][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bf16x8 f = as_bf16x8(vl[(16 * db + col) * 8 + ((4 * s + grp) ^ (col >> 1))]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) C.o[cb][db] = mfma16x16x32(f, pb[cb][s], C.o[cb][db]);
            }
        reads_ahead<1, NB>();
    };
    const int t0 = it.c * A.m + wave * A.mw;        // the wave's first row
    issue(tab.page(A, it), 0);
    C.load_q(A, it, t0, A.mw, q);
    C.begin(A, it.s, t0, A.mw);
    const Span<WIN> B(A, it.s, it.c * A.m, A.m);    // of all its rows
    for (int stg = 0;; stg ^= 1) {
        const int p0 = TILE * it.template at<WIN>(A);
        const bool more = ++it.t < end;
        const size_t at = more ? tab.page(A, it) : 0;
        // This wave's part of the tile is in LDS: vmcnt(0), by the builtin, so that the compiler knows that nothing else is
        // under way either.
        __builtin_amdgcn_s_waitcnt(0x0F70);
        __syncthreads();
        // Values that not all of the item's rows see: where some are not finite they are taken out.
        bool spoilt = false;
        if (B.edge(A, p0)) {
            uint32_t any = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x4 x = vl[stg][tid + 256 * i];
#pragma unroll
                for (int e = 0; e < 4; ++e) any |= not_finite(x[e]);
            }
            spoilt = __syncthreads_or(any);
        }
        if (spoilt) {
#pragma unroll 1
            for (int i = tid; i < D * 8; i += 256) {
                const int d = i >> 3, c = (i & 7) ^ ((d >> 1) & 7);
                u32x4 x = vl[stg][i];
                uint32_t bits = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t b = not_finite(x[e]);
                    bits |= (b >> 15 & 1) << (2 * e) | (b >> 31) << (2 * e + 1);
                    x[e] &= ~halves(b);
                }
                vl[stg][i] = x;
                ((uint8_t*)&nf[d])[c] = (uint8_t)bits;
            }
            __syncthreads();
            C.spoil(A, nf, p0);
        }
        if (more) issue(at, stg ^ 1);
        if (C.sees(A, p0)) {
            f32x4 sc[NB][4];
            scores(kl[stg], sc);
            C.maxima(A, sc, C.edge(A, p0), p0);
            bf16x8 pb[NB][2];
            C.weights(A, sc, pb);
            values(vl[stg], pb);
        }
        if (!more) break;
    }
    C.finish(A, it, t0, A.mw, P.parts == 1, A.part + ((size_t)(P.slot + P.part * P.step) * A.cols + wave * wcols) * PSTRIDE);
}

// Joins the parts of items that have several: workgroup (item, 16 of its columns); half a wave takes two columns, lane
// i dimensions 4 i .. + 3 of them, two parts requested at a time.
constexpr int kJoinPartCols = 16;
template <bool WIN>
__global__ __launch_bounds__(kJoinThreads) void join_parts_kernel(AttnArgs A) {
    Part P;
    if (!take_part<WIN>(A, blockIdx.x, true, &P)) return;
    const Item& it = P.it;
    const int np = P.parts, r = A.a / A.g, cols = min(A.cols, (it.s.n - it.c * A.m) * r);
    const int lane = threadIdx.x & 31, c0 = kJoinPartCols * blockIdx.y + 2 * (threadIdx.x >> 5);
    if (np == 1 || c0 >= cols) return;
    const float* p = A.part + (size_t)P.slot * A.cols * PSTRIDE;
    const size_t step = (size_t)P.step * A.cols * PSTRIDE;
    float M[2] = {-INFINITY, -INFINITY}, den[2] = {0.f, 0.f};
    f32x4 num[2] = {};
    for (int i0 = 0; i0 < np; i0 += 2) {
        f32x4 v[2][2];
        f32x2 ml[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // A part past the last and a column past the item's repeat the last one.
                const float* s = p + min(i0 + i, np - 1) * step + (size_t)min(c0 + j, cols - 1) * PSTRIDE;
                v[i][j] = *(const f32x4*)(s + 4 * lane);
                ml[i][j] = *(const f32x2*)(s + D);
            }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (i0 + i >= np) continue;
                const float Mn = fmaxf(M[j], ml[i][j][0]), f = __builtin_amdgcn_exp2f(M[j] - Mn), wt = __builtin_amdgcn_exp2f(ml[i][j][0] - Mn);
                den[j] = den[j] * f + wt * ml[i][j][1];
                num[j] = num[j] * f + wt * v[i][j];
                M[j] = Mn;
            }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = c0 + j, t = it.c * A.m + c / r;
        if (c >= cols) break;
        const float inv = 1.f / den[j];
        u32x2 o = {pack2bf(num[j][0] * inv, num[j][1] * inv), pack2bf(num[j][2] * inv, num[j][3] * inv)};
        if (t >= it.s.act) o = u32x2{0, 0};
        *(u32x2*)(A.out + ((size_t)(it.s.row0 + t) * A.a + it.kvh * r + c % r) * D + 4 * lane) = o;
    }
}

// Shares of the list: one wave a SIMD.
int few_shares(int simds) { return std::min(simds, kMaxDecodeSplits); }
constexpr int64_t kPieceCols = 1 << 18;      // columns of the pieces: 138 MB

constexpr int kFewCols = 32;      // up to here a wave takes all columns of an item
template <int NB, bool WIN>
void launch_few(int nw, int grid, const AttnArgs& A, hipStream_t st) {
    if (nw == 0) hipLaunchKernelGGL((rows_few_kernel<0, NB, WIN>), dim3(grid), dim3(64), 0, st, A);
    else if (nw == 1) hipLaunchKernelGGL((rows_few_kernel<1, NB, WIN>), dim3(grid), dim3(64), 0, st, A);
    else if (nw == 2) hipLaunchKernelGGL((rows_few_kernel<2, NB, WIN>), dim3(grid), dim3(128), 0, st, A);
    else hipLaunchKernelGGL((rows_few_kernel<4, NB, WIN>), dim3(grid), dim3(256), 0, st, A);
}

// Waves that take an item of few columns (16 nb) where one launch without a join is the faster one, else 0.  tiles: of the
// longest item.  One workgroup an item of 1, 2 and 4 waves against two launches (the list, or equal parts), 32 heads on 8, in us.
// nb 1: 1 sequence of 200 positions 8.4, 7.9, 7.7 and 9.4, of 500 13.5, 11.2, 11.0 and 9.5; 8 of 200 9.2, 8.2, 7.8 and 9.2, 500
// 16, 11.9, 11.6 and 9.7; 16 of 500 16.7, 12.2, 11.8 and 12.3, 1000 31, 20, 19.5 and 17.8; 32 of 1000 39, 28, 27 and 31, 2000 74,
// 50, 49 and 53; 64 of 500 26.6, 27.3, 30 and 31.6, 2000 91, 94, 95 and 99; 100 of 500 44, 47, 53 and 51, 2000 165, 159, 169 and
// 156.  nb 2 (8 rows a sequence): 1 of 500 17.9, 15.9, 14.7 and 10.5; 8 of 500 19.8, 16.9, 15.4 and 13.1; 16 of 1000 38, 26, 22.4
// and 23.3; 64 of 1000 52, 56, 60 and 67.  The rule takes the slower one at three of these: 8 of 500 (4 waves, 20 %), 32 of 2000
// (the list, 8 %) and 100 of 2000 (1 wave, 5 %).  (Past 32 tiles one long sequence among short ones would cost more than there is
// to gain; 8 waves have too few registers: 18.9 for 1 of 500, nb 2.)
int few_waves(int64_t items, int64_t tiles, int nb, int simds) {
    if (tiles > std::min<int64_t>(32, nb == 1 ? 4 + items / 11 : items < 96 ? 4 : 32)) return 0;
    return items <= simds / 4 ? 4 : items < simds / 2 ? 2 : 1;
}

// How many columns are cut: columns of a wave, and the parts of items, by what the launch would take, in us.
//
// t1: a tile of a workgroup that has its CU to itself, t2: one of two workgroups'.  A launch takes, whichever is most (and above
// it where they are alike), its longest part, all tiles on all CUs, or K and V from memory once; of parts that are alike, the
// rounds of them that the device runs.  Every round begins some parts, and pieces go to memory and back.  What the host has
// are bounds: of several sequences 0.79 of the longest's tiles counts, and the longest parts may come last (not of prompts
// without a context, of which the longest begin).
//
// Parts by length (no more than a bound of each sequence's tiles says) cost nothing to find; parts by count, which the device
// cuts from what the sequences really have, about 5 us more, and need no room for pieces that are not made.  Neither is
// better throughout.  The constants are fitted to sweeps over such launches on one card, most of them of 32 heads on 8; equal
// contexts of several sequences and one long among short ones come out 10 to 20 % from the best.  Measured, the best of 1, 2
// and 3 blocks of 16 columns: whole, parts by length, by count; 32 heads on 8.  Alike: a prompt of 2000 rows 49, 60, 58; 4
// prompts of 1000 51, 92, 72; 600 rows behind 3000 positions 64, 50, 59; 100 behind 30000 446, 74, 75; 400 behind 30000 448,
// 214, 198; 8 x 100 behind 3000 67, 62, 72.  Unlike: 4 x 100-800 behind 0-3000 96, 82, 68; 3 x 333-1001 behind 700-5000 147,
// 118, 120; 3 x 50-500 behind 100-20000 321, 120, 101; 16 x 9-200 behind 10-6000 153, 121, 109; 2 x 300-2000 behind
// 1000-40000 (64 heads) 1201, no room, 571.
struct Cut {
    int nb = 0, longest = 0, parts = 0, jobs = 0, grid = 0, m = 0, cols = 0, slots = 0;
    int64_t items = 0, sparse = 0, most = 0;      // a bound of the items, and with every sequence as long as the longest
    double us = 0;
    Cut() = default;
    Cut(int nb_, int heads, const AttnArgs& A_, int simds, bool window)
        : nb(nb_), A(&A_), cus(std::max(simds / 4, 1)), win(window) {
        const NewRows& r = A->r;
        m = 4 * std::min(16 * nb / heads, (r.max_new + 3) / 4);
        cols = m * heads;
        slots = 2 * cus;
        items = (int64_t)A->g * (r.rows / m + r.B);
        sparse = (int64_t)A->g * r.B * ((r.max_new + m - 1) / m);
    }
    void by_length(int k, Cut* best) {
        longest = (int)((most + k - 1) / k);
        parts = (int)((most + longest - 1) / longest);
        jobs = 0;
        if (sparse * parts >= 1 << 24 || (parts > 1 && items * parts * cols > kPieceCols)) return;      // 2^32 threads
        grid = (int)(sparse * parts);
        take(best);
    }
    void by_count(int count, Cut* best) {
        parts = 0;
        jobs = count;
        if (items >= jobs || sparse > INT32_MAX || (int64_t)jobs * cols > kPieceCols) return;
        grid = jobs;
        take(best);
    }

private:
    const AttnArgs* A = nullptr;
    int cus = 1;
    bool win = false;
    void take(Cut* best) {
        static constexpr double t1s[3] = {0.75, 1.14, 1.38}, t2s[3] = {0.57, 0.85, 1.26};
        const NewRows& r = A->r;
        const double t1 = t1s[nb - 1], t2 = t2s[nb - 1], n = (double)most;
        double mean = win ? std::max(n - 1, 1.) : std::max(n - r.max_new / (2. * TILE), n / 2);
        const bool like = win || mean > 0.8 * n, several = r.B > 1;
        const double part = several ? 0.79 : 1.;
        if (!win) mean *= part;
        const double N = several ? std::min(A->g * ((double)r.rows / m + 0.5 * r.B), (double)sparse) : sparse, T = N * mean;
        const double L = jobs ? std::ceil(T / std::max(jobs - N, 1.)) : longest;
        const double n_parts = N * std::max(1., mean / L) + (mean > L && several ? 0.34 * N : 0);
        const double all = T * t2 / cus, once = part * A->g * r.B * n * (4. * kHalfPage / 6e6);
        const double rounds = n_parts / slots, full = std::floor(rounds), rest = rounds - full;
        const double last = rest == 0 ? 0 : rest <= 0.5 ? t1 : t1 + (2 * t2 - t1) * (2 * rest - 1);
        const double even = T / n_parts * (2 * t2 * full + last), longest_us = std::min(L, n) * t1;
        const double u = like && (!jobs || !several) ? 0.55 : 0.1;
        us = 5 + (1 - u) * std::cbrt(longest_us * longest_us * longest_us + all * all * all + once * once * once) +
             u * std::max(even, std::max(longest_us, once)) + 3.4 * std::ceil(rounds) + grid / 2000.;
        if (parts != 1) us += 3 + n_parts * cols * (PSTRIDE * 4 * 0.4e-6);
        if (jobs) us += 4.8;
        if (several && n * TILE >= r.max_new + TILE) us += (jobs ? 0.1 : 0.68) * std::min(L, n) * t2;     // cached contexts
        if (!best->nb || us < best->us) *best = *this;
    }
};

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
    hipError_t e;
    if (r.max_new * heads <= kFewCols) {
        A.m = r.max_new;
        A.cols = A.m * heads;
        // The list counts tiles in 31 bits; where it might not, items run one by one.
        const int items = r.B * A.g, nw = items * most(A.m) <= INT32_MAX ? few_waves(items, most(A.m), A.cols <= 16 ? 1 : 2, simds) : 1;
        if (nw) {
            if (A.cols <= 16) launch_few<1, WIN>(nw, items, A, st);
            else launch_few<2, WIN>(nw, items, A, st);
            return hipGetLastError();
        }
        const int shares = few_shares(simds);
        A.cut = (int2*)(A.part + (size_t)2 * shares * A.cols * PSTRIDE);
        // Items in equal parts, which need no search in the list, where the shares' lengths are alike all the same: of one
        // sequence, or where there is a share for every tile (1 sequence of 4000 positions 11.3 us, listed 11.8, of 16000 19.3 and
        // 19.9; 8 rows behind 977 10.8 and 11.7; below 2000 positions both wait for the host's two launches).
        int grid = shares;
        if (items <= shares && (r.B == 1 || items * most(A.m) <= shares)) {
            A.parts = (int)std::min<int64_t>(shares / items, most(A.m));
            grid = items * A.parts;
        }
        if (A.cols <= 16) launch_few<1, WIN>(0, grid, A, st);
        else launch_few<2, WIN>(0, grid, A, st);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        // Few pieces an item, a wave a column; many, four waves.
        if (shares <= 32 * items)
            hipLaunchKernelGGL(join_short_kernel, dim3((items * A.cols + kJoinWaves - 1) / kJoinWaves), dim3(kJoinThreads), 0, st, A);
        else
            hipLaunchKernelGGL(join_few_kernel, dim3(items * A.cols), dim3(kJoinThreads), 0, st, A);
        return hipGetLastError();
    }
    Cut best;
    for (int nb = 1; nb <= 3; ++nb) {
        if (std::min(16 * nb / heads, (r.max_new + 3) / 4) < 1) continue;
        Cut c(nb, heads, A, simds, WIN);
        c.most = most(c.m);
        for (int k = 1; k <= std::min<int64_t>(64, c.most); k += 1 + k / 6) c.by_length(k, &best);
        if (c.most >= 8)
            for (int k = 1; k <= 4; ++k) c.by_count(k * c.slots, &best);
    }
    if (!best.nb) {
        // The longest sequence's blocks times B are more than a grid can have: no item is cut.
        for (int nb = 1; nb <= 3; ++nb)
            if (std::min(16 * nb / heads, (r.max_new + 3) / 4) >= 1) best = Cut(nb, heads, A, simds, WIN);
        best.jobs = 1;
        best.grid = best.items;
        if (best.items >= 1 << 24 || best.sparse > INT32_MAX) return hipErrorInvalidValue;
    }
    A.mw = best.m / 4;
    A.m = best.m;
    A.cols = best.cols;
    A.longest = best.longest;
    A.parts = best.parts;
    A.jobs = best.jobs;
    if (best.nb == 1) hipLaunchKernelGGL((rows_many_kernel<1, WIN>), dim3(best.grid), dim3(256), 0, st, A);
    else if (best.nb == 2) hipLaunchKernelGGL((rows_many_kernel<2, WIN>), dim3(best.grid), dim3(256), 0, st, A);
    else hipLaunchKernelGGL((rows_many_kernel<3, WIN>), dim3(best.grid), dim3(256), 0, st, A);
    if ((e = hipGetLastError()) != hipSuccess || best.parts == 1 || best.jobs == 1) return e;
    const dim3 join(best.jobs ? best.items : best.sparse, (A.cols + kJoinPartCols - 1) / kJoinPartCols);
    hipLaunchKernelGGL((join_parts_kernel<WIN>), join, dim3(kJoinThreads), 0, st, A);
    return hipGetLastError();
}

}  // namespace

// Pieces, then what the few columns' join reads.
size_t attention_rows_bytes(int B, int g, int simds) {
    const size_t cols = std::max<size_t>(kPieceCols, (size_t)2 * kFewCols * few_shares(simds));
    return cols * PSTRIDE * sizeof(float) + (size_t)B * g * sizeof(int2);
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
