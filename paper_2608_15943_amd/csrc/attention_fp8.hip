// Attention of a call's new rows over the 8-bit paged cache: one new token a sequence, a few, or
// a whole prompt; row i of sequence b sits at position len_b + i and sees positions [0, len_b + i].
//
// The rows of a sequence and the r = a / g query heads of a K/V head are the columns of one
// product.  A wave takes 16 or 32 of them over the 64-position tiles (a page each) of their K/V head,
// each once, with the running maximum and sum of the softmax; codes are widened to bf16 in
// registers (exactly: e4m3 has 4 significant bits) and multiplied on v_mfma_f32_16x16x32_bf16.
//
//   S^T = K Q^T  Row rho of score block tb is position 16 (rho / 4) + 4 tb + rho % 4 of the tile, so
//                that lane group grp ends with positions 16 grp .. 16 grp + 15: one scale block, and
//                the run that the second product sums over.  The K scale multiplies a lane's
//                scores, one factor for all of them.
//   O^T += V^T P^T  The V scale, a power of two, goes into the exponent of P before P is rounded to
//                bf16 (8 bits), the type of the product beside V's codes; the sum of the weights is
//                taken from the rounded P, so that its rounding cancels where it is common.  It
//                leaves 0.0021-0.0024 of the output's scale as the error against 64 bits, where the
//                output's own rounding is 0.0016-0.0017.
//
// attention_few_kernel: sequences with at most 32 columns (single tokens, a few proposed ones); K and V go straight
// to registers.  Bound by reading the cache: 64 x 32768 positions (32 heads on 8, 4.3 GB) 707 us, 6.1 TB/s; 8 x
// 64K-128K 276 us, 5.9 TB/s.  attention_many_kernel: more columns; four waves share each tile through LDS.  Bound by
// the vector instructions (widening, softmax) beside the matrix ones: prompts of 4 x 4096 rows (16 heads on 8) 263 us,
// 1045 TFLOP/s, once the clock has risen (330 us in the first 20 calls).
//
// Work: the tiles of all items (a sequence's block of rows and a K/V head) in one list, in the order
// (sequence, K/V head, block, tile), which the waves (workgroups) share evenly: an item that begins
// and ends with one of them is written by it, the others leave their pieces (running maximum, sum,
// unnormalised O) to a second kernel.  Where contexts are short or items many, items run one by one
// instead, in one launch: of few columns on workgroups of 1, 2 or 8 waves, which join in LDS, of many the longest
// first.
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

struct CutItem {
    int np, row, n, act, head, pad[3];     // pieces; first row in the tensors, rows (of them act see something), first head
};

struct AttnArgs {
    NewRows r;
    const uint16_t* q;
    const uint8_t* kc;
    const uint8_t* vc;
    const float* sc;
    uint16_t* out;
    float* part;       // [2 W][cols][PSTRIDE]: slot 2 w: share w's piece of an item that began before it,
                       // 2 w + 1: of one that begins with it and goes on
    int a, g;
    int m, cols;       // rows of an item, columns that they make
    int mw;            // rows of a wave of attention_many_kernel: m / 4
    // What the join reads: of attention_few_kernel, for each sequence and K/V head the share that
    // begins it and how many shares have a part; of attention_many_kernel, for each share the item that it
    // begins and does not end (np 0: none).
    int2* cut;
    struct CutItem* cut_many;
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
// FEW: every sequence has one block at most.
template <bool FEW>
__device__ __forceinline__ uint32_t seq_tiles(const SeqRows& s, int m) {
    if (FEW) return s.n ? tiles_of(s, m, 0) : 0;
    return tiles_before(s, m, blocks_of(s, m));
}

// The list shared by W waves: wave w starts at tile floor(w T / W).  T < 2^31, W <= 4096.
struct Split {
    uint32_t T, W, q, rem;
    Split() = default;
    __device__ __forceinline__ Split(uint32_t T_, uint32_t waves) : T(T_), W(min(T_, waves)), q(T_ / max(W, 1u)), rem(T_ % max(W, 1u)) {}
    __device__ __forceinline__ uint32_t start(uint32_t w) const { return w * q + w * rem / W; }
    // The wave that holds tile x: ceil((x + 1) W / T) - 1; exact in double.
    __device__ __forceinline__ uint32_t wave_of(uint32_t x) const {
        return (uint32_t)(((double)(x + 1) * (double)W - 1.0) / (double)T);
    }
};

// 64 sequences at a time, one a lane: their rows, tiles for one K/V head, and the tiles of the list
// before each.
template <bool FEW>
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
            n = seq_tiles<FEW>(s, A.m);
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
template <bool FEW>
__device__ __forceinline__ uint32_t list_tiles(const AttnArgs& A, Lanes<FEW>& L) {
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
template <bool FEW>
__device__ __forceinline__ Item find_tile(const AttnArgs& A, Lanes<FEW>& L, uint32_t x) {
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
    it.c = 0;
    it.t = rem;
    if (!FEW) {
        // The last block with tiles_before <= rem.  About c (1 + (len + m / 2) / 64) + c^2 m / 128 tiles lie
        // before block c: its root, then exactly.
        const float al = A.m / 128.f, be = 1.f + (max(it.s.len, 0) + 0.5f * A.m) / 64.f;
        const int cmax = blocks_of(it.s, A.m) - 1;
        int c = (int)((sqrtf(be * be + 4.f * al * rem) - be) / (2.f * al));
        c = __builtin_amdgcn_readfirstlane(min(max(c, 0), cmax));
        uint32_t n0 = tiles_before(it.s, A.m, c);
        while (c > 0 && n0 > rem) n0 -= tiles_of(it.s, A.m, --c);
        for (; c < cmax; ++c) {
            const uint32_t k = tiles_of(it.s, A.m, c);
            if (n0 + k > rem) break;
            n0 += k;
        }
        it.c = c;
        it.t = rem - n0;
    }
    it.n = tiles_of(it.s, A.m, it.c);
    return it;
}

// Whether the sequences have no more rows together than the call has, as the launch's rule takes it for the bound of the
// list's 2^31 tiles (of few columns it holds whatever the offsets are).  Exact: rows < 2^23, 384 or more values each.
__device__ __forceinline__ bool rows_bounded(const NewRows& r) {
    float n = 0.f;
    for (int b = threadIdx.x & 63; b < r.B; b += 64) n += (float)seq_rows(r, b).n;
    return wave_sum(n) <= (float)r.rows;
}

// A share of the list: where it begins and ends.
template <bool FEW>
__device__ __forceinline__ bool take_share(const AttnArgs& A, Split* sp, uint32_t* w, uint32_t* left, Item* it) {
    Lanes<FEW> L;
    const bool bounded = FEW || rows_bounded(A.r);
    *sp = Split(list_tiles(A, L), gridDim.x);
    if (!bounded || blockIdx.x >= sp->W) return false;
    // Shares in one block on one XCD: neighbours read the same K/V head.
    *w = xcd_remap(blockIdx.x, sp->W);
    const uint32_t x = sp->start(*w);
    *left = sp->start(*w + 1) - x;
    *it = find_tile(A, L, x);
    return true;
}
// The item behind `it` in the list; false past the end.
__device__ __forceinline__ bool next_item(const AttnArgs& A, Item& it) {
    it.t = 0;
    if (++it.c == blocks_of(it.s, A.m)) {
        it.c = 0;
        if (++it.kvh == A.g) {
            it.kvh = 0;
            for (++it.b; it.b < A.r.B; ++it.b) {       // sequences without rows have no tiles
                it.s = seq_rows(A.r, it.b);
                if (it.s.n) break;
            }
            if (it.b >= A.r.B) return false;
        }
    }
    it.n = tiles_of(it.s, A.m, it.c);
    return true;
}

// Index of the page of tile it.t, for it.kvh.  A wave keeps 64 entries of a table row, so that one
// dependent load serves 64 tiles.
struct Table {
    int b = -1, c = -1, v = 0;
    __device__ __forceinline__ size_t page(const AttnArgs& A, const Item& i) {
        if (i.b != b || (i.t >> 6) != c) {
            b = i.b;
            c = i.t >> 6;
            const int e = 64 * c + (threadIdx.x & 63);
            v = e < A.r.stride ? A.r.pt[(size_t)i.b * A.r.stride + e] : 0;
        }
        const int pg = min(max(__builtin_amdgcn_readlane(v, i.t & 63), 0), A.r.n_pages - 1);
        return (size_t)i.kvh * A.r.n_pages + pg;
    }
};

// The thread's index, unknown to the compiler: what is computed from it where an item begins or ends is not
// held in registers (or spilled) through the loop over its tiles.
__device__ __forceinline__ int thread_now() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// 16 NB columns of an item, from row t0 of the sequence on: a lane's column of block cb is head tj of
// row t0 + tc.
template <int NB>
struct Columns {
    int lim[NB];             // the last position that the column sees, -1 where there is none
    float m[NB], l[NB];      // running maximum (log2 domain) and sum of the weights
    f32x4 o[NB][8];          // O^T: dimensions 16 db + 4 grp + 0..3 of the column
    int all, last;           // positions up to `all` every row sees, past `last` none does

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
    // Dimensions 16 grp .. + 15 (j = 0) and 64 + 16 grp .. + 15 (j = 1) of the query of column cb, in two words
    // of 8 each: the order of the K codes' 16-byte runs.
    static __device__ __forceinline__ void load_q(const AttnArgs& A, const Item& it, int t0, int rows, int cb, u32x4 (&v)[2][2]) {
        const int grp = (thread_now() >> 4) & 3, r = A.a / A.g;
        const bool real = limit(it.s, t0, rows, r, cb) >= 0;
        const size_t row = it.s.row0 + (real ? t0 + row_of(cb, rows, r) : 0);
        const uint16_t* p = A.q + (row * A.a + it.kvh * r + head_of(cb, r)) * D + 16 * grp;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v[j][h] = u32x4{0, 0, 0, 0};
                if (real) v[j][h] = *(const u32x4*)(p + 64 * j + 8 * h);
            }
    }
    // Begins rows t0 .. t0 + rows - 1 of a sequence (their queries are loaded).
    __device__ __forceinline__ void begin(const SeqRows& s, int t0, int rows, int r) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            lim[cb] = limit(s, t0, rows, r, cb);
            m[cb] = kNoScore;
            l[cb] = 0.f;
#pragma unroll
            for (int db = 0; db < 8; ++db) o[cb][db] = f32x4{};
        }
        const int n = min(s.act - t0, rows);
        all = n > 0 ? s.len + t0 : -1;
        last = n > 0 ? s.len + t0 + n - 1 : -1;
    }
    // Weights of a tile from its scores: lane (column, grp) holds positions p0 + 4 tb + i, whose scales
    // are ks (times the score factor and, qs[cb], the column's) and vs; out: the rows of P, pb.  edge: some column does not see all
    // of the tile (branches around the masks: two copies of this code would not fit the registers).
    __device__ __forceinline__ void softmax(f32x4 (&sc)[NB][4], bool edge, int p0, float ks_, const float (&qs)[NB], float vs,
                                            bf16x8 (&pb)[NB][2]) {
        // The scales of blocks that no column sees may hold anything.
        if (edge && p0 > last) ks_ = vs = 1.f;
        // P 2^e for a V scale of 2^e >= 2^-100: weights down to 2^-26 of the largest stay normal numbers.
        const int e = (int)(__float_as_uint(vs) >> 23) - 127;
        const float vexp = vs == vs ? (float)e : vs;
        const float vinv = vs == vs ? __uint_as_float((uint32_t)(127 - e) << 23) : 1.f;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            if (edge) {
#pragma unroll
                for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (p0 + 4 * tb + i > lim[cb]) sc[cb][tb][i] = -INFINITY;
            }
            const float ks = ks_ * qs[cb];
            float mx = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[cb][tb][i]);
            const float mt = pair32_max(pair16_max(mx * ks));
            if (__any(mt > m[cb] + kLazy)) {
                const float m_new = fmaxf(m[cb], mt);
                const float alpha = __builtin_amdgcn_exp2f(m[cb] - m_new);
                m[cb] = m_new;
                l[cb] *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db) o[cb][db] *= alpha;
            }
            const float sub = vexp - m[cb];
            uint32_t pw[8];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[cb][tb][i] = __builtin_amdgcn_exp2f(fmaf(sc[cb][tb][i], ks, sub));
#pragma unroll
            for (int i = 0; i < 8; ++i) pw[i] = pack2bf(sc[cb][i >> 1][2 * (i & 1)], sc[cb][i >> 1][2 * (i & 1) + 1]);
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
            l[cb] += lt * vinv;
            pb[cb][0] = as_bf16x8(u32x4{pw[0], pw[1], pw[2], pw[3]});
            pb[cb][1] = as_bf16x8(u32x4{pw[4], pw[5], pw[6], pw[7]});
        }
    }
    // Masks of the words of a lane's V runs at an edge: codes past `last` (never written, perhaps) must be
    // finite, and count as 0.
    __device__ __forceinline__ uint32_t v_mask(int p0, int word) const {
        const int k = last + 1 - p0 - 4 * word;       // bytes of the word that are seen
        return k >= 4 ? 0xFFFFFFFFu : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
    }
    // The end of an item (or of a share inside it): out, or a piece.
    __device__ __forceinline__ void finish(const AttnArgs& A, const Item& it, int t0, int rows, bool whole, float* piece) {
        const int grp = (thread_now() >> 4) & 3, col = thread_now() & 15, r = A.a / A.g;
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            const float lsum = pair32_sum(pair16_sum(l[cb]));
            const int t = row_of(cb, rows, r);
            if (t >= it.s.n - t0) continue;
            if (whole) {
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
template <int NW, int NB>
__global__ __launch_bounds__(NW ? 64 * NW : 64, 2) void attention_few_kernel(AttnArgs A) {
    constexpr bool LIST = NW == 0;
    constexpr int STEP = LIST ? 1 : NW;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    Item it;
    Split sp;
    uint32_t w = 0, left;
    if constexpr (LIST) {
        if (!take_share<true>(A, &sp, &w, &left, &it)) return;
    } else {
        it.b = blockIdx.x / A.g;
        it.kvh = blockIdx.x % A.g;
        it.s = seq_rows(A.r, it.b);
        if (!it.s.n) return;
        it.c = 0;
        it.t = wave;
        it.n = tiles_of(it.s, A.m, 0);
        left = max(it.n - wave + NW - 1, 0) / NW;
    }
    Columns<NB> C;
    u32x4 q[NB][2][2];
    const int r = A.a / A.g;
    Table tab;
    u32x4 k[4][2], v[8];         // [score block][64-dimension half], [16-dimension block]
    float ks, vs;                // scales of the lane group's 16 positions
    const uint32_t koff = (16 * (col >> 2) + (col & 3)) * D + 16 * grp, voff = grp * kBlkBytes + col * kBlk;
    auto load_k = [&](size_t at) {
        const uint8_t* p = A.kc + at * kPageBytes8;
        ks = (A.sc + at * 2 * kPageBlks)[(uint32_t)grp];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int j = 0; j < 2; ++j) k[tb][j] = *(const u32x4*)(p + 4 * tb * D + 64 * j + koff);
    };
    auto load_v = [&](size_t at) {
        const uint8_t* p = A.vc + at * kPageBytes8;
        vs = (A.sc + at * 2 * kPageBlks + kPageBlks)[(uint32_t)grp];
#pragma unroll
        for (int db = 0; db < 8; ++db) v[db] = *(const u32x4*)(p + 16 * db * kBlk + voff);
    };
    auto load_q = [&](const Item& i) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) C.load_q(A, i, i.c * A.m, A.m, cb, q[cb]);
    };
    float one[NB];
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) one[cb] = 1.f;
    bool whole = !LIST || it.t == 0;        // the share has the item from its first tile on
    uint32_t x = LIST ? sp.start(w) : 0;      // the list's tile
    auto begin = [&](const Item& i) {
        C.begin(i.s, i.c * A.m, A.m, r);
        if (LIST && whole && lane == 0) A.cut[i.b * A.g + i.kvh] = make_int2(w, sp.wave_of(x + i.n - 1) - w + 1);
    };
    load_q(it);
    begin(it);
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
                more = next_item(A, nx);
            else
                nx.t += STEP;
        }
        const size_t at = more ? tab.page(A, nx) : 0;
        const int p0 = TILE * it.t + 16 * grp;
        const bool edge = TILE * it.t + TILE - 1 > C.all;
        f32x4 sc[NB][4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bf16x8 f = widen(k[tb][s >> 1][2 * (s & 1)], k[tb][s >> 1][2 * (s & 1) + 1]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb)
                    sc[cb][tb] = mfma16x16x32(f, as_bf16x8(q[cb][s >> 1][s & 1]), s ? sc[cb][tb] : f32x4{});
            }
        const float kf = ks * A.scale_log2;
        __builtin_amdgcn_sched_barrier(0);
        // A part of a tile (and the queries) is requested again as soon as it has been multiplied: 16
        // KB a wave are always under way, without a second set of registers.
        if (more) {
            load_k(at);
            if (ends) load_q(nx);
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pb[NB][2];
        C.softmax(sc, edge, p0, kf, one, vs, pb);
        if (edge) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t mask = C.v_mask(p0, i);
#pragma unroll
                for (int db = 0; db < 8; ++db) v[db][i] &= mask;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 f = widen(v[db][2 * h], v[db][2 * h + 1]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) C.o[cb][db] = mfma16x16x32(f, pb[cb][h], C.o[cb][db]);
            }
        __builtin_amdgcn_sched_barrier(0);
        if (more) load_v(at);
        if (NW > 1 && !more) break;
        if (ends || !more) {
            C.finish(A, it, it.c * A.m, A.m, whole && ends, A.part + (2 * (size_t)w + (whole ? 1 : 0)) * A.cols * PSTRIDE);
            if (!more) break;
            whole = true;
            ++x;
            begin(nx);
            --x;
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
            for (int v = 0; v < NW; ++v) M = fmaxf(M, parts[v][c][D]);
#pragma unroll
            for (int v = 0; v < NW; ++v) {
                const float f = __builtin_amdgcn_exp2f(parts[v][c][D] - M);
                den += f * parts[v][c][D + 1];
                num += f * *(const f32x2*)&parts[v][c][2 * lane];
            }
            const uint32_t o = c / r < it.s.act ? pack2bf(num[0] / den, num[1] / den) : 0u;
            *(uint32_t*)(A.out + ((size_t)(it.s.row0 + c / r) * A.a + it.kvh * r + c % r) * D + 2 * lane) = o;
        }
    }
}

typedef __attribute__((address_space(3))) void lvoid_t;

// Buffer resource of `bytes` bytes at p, the same for the wave (word 3: a valid 32-bit data format).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes) {
    const uint64_t a = (uint64_t)p;
    const uint64_t u = (uint32_t)__builtin_amdgcn_readfirstlane((int)a) |
                       (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32;
    return __builtin_amdgcn_make_buffer_rsrc((void*)u, 0, bytes, 0x00020000);
}

// The queries of a wave's columns as sums of an e4m3 and an e5m2 number, times a power of two s for each column: the
// 8 significant bits of bf16 in 4 and what 4 bits leave.  Scores are then products of 8-bit numbers as they are in
// memory, K with both halves, at twice the rate of bf16 and without widening K.
//
// In units of s the column's largest value lies in (224, 448].  From 2^-6 on hi takes 4 of a value's 8 bits and leaves
// j units of the last of them, |j| <= 8: 3 bits, a number of e5m2, so that the sum is exact.  Below, hi is a multiple of
// 2^-9 and leaves 2^-10 at most, of which lo, with 3 bits, misses 2^-14 at most: 2^-21.8 of the column's largest value, or 2^-114
// where s is 2^-100, its least.  (lo in e4m3 would miss up to 2^-10 there, 2^-17.8 of the largest value.)
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int NB>
struct Queries8 {
    i32x8 hi[NB], lo[NB];
    float s[NB];
    __device__ __forceinline__ void load(const AttnArgs& A, const Item& it, int t0, int rows) {
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            u32x4 v[2][2];
            Columns<NB>::load_q(A, it, t0, rows, cb, v);
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        m = max(m, max((v[j][h][i] << 16) & 0x7FFFFFFFu, v[j][h][i] & 0x7FFF0000u));
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            s[cb] = e4m3_scale(m);
            const float inv = 1.f / s[cb];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t a = v[j][h][2 * i], b = v[j][h][2 * i + 1];
                        const float x0 = __uint_as_float(a << 16) * inv, x1 = __uint_as_float(a & 0xFFFF0000u) * inv,
                                    x2 = __uint_as_float(b << 16) * inv, x3 = __uint_as_float(b & 0xFFFF0000u) * inv;
                        const uint32_t c = e4m3_pack(x0, x1, x2, x3);
                        const f32x2 y0 = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), y1 = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
                        hi[cb][4 * j + 2 * h + i] = (int)c;
                        const int r = __builtin_amdgcn_cvt_pk_bf8_f32(x0 - y0[0], x1 - y0[1], 0, false);
                        lo[cb][4 * j + 2 * h + i] = __builtin_amdgcn_cvt_pk_bf8_f32(x2 - y1[0], x3 - y1[1], r, true);
                    }
        }
    }
};
// a in e4m3, b in e4m3 or (B 1) e5m2.
template <int B>
__device__ __forceinline__ f32x4 mfma_8bit(i32x8 a, i32x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, B, 0, 0, 0, 0);
}

// N 16-byte LDS reads at addr (or a0, a1 in turn) + OFF, STEP apart, and their wait: written by hand, since
// the compiler would first wait for the loads that go into the other stage.
template <int OFF, int STEP>
__device__ __forceinline__ void lds_pairs(uint32_t a0, uint32_t a1, u32x4 (&f)[4]) {
    asm volatile("ds_read_b128 %0, %4 offset:%6\n\tds_read_b128 %1, %5 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\t"
                 "ds_read_b128 %3, %5 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                 : "v"(a0), "v"(a1), "i"(OFF), "i"(OFF + STEP)
                 : "memory");
}
template <int OFF, int STEP>
__device__ __forceinline__ void lds_run(uint32_t a, u32x4 (&f)[4]) {
    asm volatile("ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\t"
                 "ds_read_b128 %3, %4 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                 : "v"(a), "i"(OFF), "i"(OFF + STEP), "i"(OFF + 2 * STEP), "i"(OFF + 3 * STEP)
                 : "memory");
}

// Workgroup: an item of 4 mw rows, wave v's 16 NB columns are its rows v mw .. (v + 1) mw - 1.  The tiles
// go from memory to LDS directly, two stages of 16 KB, one barrier a tile: it ends the loads of the
// tile that comes and the reads of the one before it, whose stage is then loaded again.  Three (NB 1:
// four) workgroups a CU run in each other's waits.
// LIST: a share of the list; else one item, counted from a sequence's last.
template <bool LIST, int NB>
__global__ __launch_bounds__(256, NB == 1 ? 4 : 3) void attention_many_kernel(AttnArgs A) {
    // K rows of 8 chunks of 16 bytes: chunk c of row R at place c ^ key(R), so that the 16 rows of a
    // fragment read (R % 4 and R / 16 run) fall on all banks; V as it is in memory.
    __shared__ u32x4 kl[2][512], vl[2][512];
    auto key = [](int R) { return ((R >> 1) & 1) | (((R >> 4) & 3) << 1); };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    Item it;
    uint32_t w = 0, left;
    if constexpr (LIST) {
        Split sp;
        if (!take_share<false>(A, &sp, &w, &left, &it)) {
            if (tid == 0) A.cut_many[blockIdx.x].np = 0;
            return;
        }
        // The item that the share begins and does not end: that of its last tile.
        if (tid < 64) {
            CutItem cut{};
            if (w + 1 < sp.W) {
                const uint32_t xe = sp.start(w + 1) - 1;
                Lanes<false> L;
                list_tiles(A, L);
                const Item e = find_tile(A, L, xe);
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
        it.n = tiles_of(it.s, A.m, it.c);
        left = it.n;
    }
    const int r = A.a / A.g, wcols = A.mw * r;
    Columns<NB> C;
    Queries8<NB> Q;
    Table tab;
    float kn, vn;          // scales of the tile that comes
    auto issue = [&](const Item& i, int stg) {
        const size_t at = tab.page(A, i);
        // Buffer resources of the two pages: a lane's address is one offset.
        const __amdgpu_buffer_rsrc_t kr = buffer_of(A.kc + at * kPageBytes8, kPageBytes8),
                                     vr = buffer_of(A.vc + at * kPageBytes8, kPageBytes8);
        const __amdgpu_buffer_rsrc_t sr = buffer_of(A.sc + at * 2 * kPageBlks, 2 * kPageBlks * sizeof(float));
        // The lane's 16 bytes of the first of this wave's two KB of K and V (the second's key is the same).
        const int now = thread_now() & 63;
        const uint32_t ksrc = (now >> 3) * D + 16 * ((now & 7) ^ ((now >> 4) & 1) ^ (2 * wave)), vsrc = 16 * now, ssrc = 4 * (now >> 4);
        kn = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sr, ssrc, 0, 0));
        vn = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sr, ssrc, 4 * kPageBlks, 0));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lvoid_t*)&kl[stg][128 * wave + 64 * i], 16, ksrc, 2048 * wave + 1024 * i, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lvoid_t*)&vl[stg][128 * wave + 64 * i], 16, vsrc, 2048 * wave + 1024 * i, 0, 0);
        }
    };
    bool whole = it.t == 0;
    int t0 = it.c * A.m + wave * A.mw;        // the wave's first row
    issue(it, 0);
    Q.load(A, it, t0, A.mw);
    C.begin(it.s, t0, A.mw, r);
    for (int stg = 0;; stg ^= 1) {
        const bool ends = it.t + 1 == it.n;
        bool more = left > 1;
        Item nx = it;
        if (more) {
            if (LIST && ends)
                more = next_item(A, nx);
            else
                ++nx.t;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wave's part of the tile is in LDS
        __syncthreads();
        const float ks = kn * A.scale_log2, vs = vn;
        if (more) issue(nx, stg ^ 1);
        const int p0 = TILE * it.t + 16 * grp;
        if (TILE * it.t <= C.last) {          // the wave's rows see some of it
            const bool edge = TILE * it.t + TILE - 1 > C.all;
            f32x4 sc[NB][4];
            // The lane's K chunks of the two dimension halves (key(R) is the same for its four rows R).
            const int now = thread_now(), krow = 16 * ((now >> 2) & 3) + (now & 3);
            const uint32_t ka0 = (uint32_t)(uintptr_t)&kl[stg][krow * 8 + (((now >> 4) & 3) ^ key(krow))], ka1 = ka0 ^ 64;
            auto scores = [&](auto tb_t) __attribute__((always_inline)) {
                constexpr int tb0 = decltype(tb_t)::value;
                u32x4 kv[4];
                lds_pairs<tb0 * 4 * D, 4 * D>(ka0, ka1, kv);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x4 x = kv[2 * i], y = kv[2 * i + 1];
                    const i32x8 f = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
#pragma unroll
                    for (int cb = 0; cb < NB; ++cb) sc[cb][tb0 + i] = mfma_8bit<0>(f, Q.hi[cb], f32x4{});
#pragma unroll
                    for (int cb = 0; cb < NB; ++cb) sc[cb][tb0 + i] = mfma_8bit<1>(f, Q.lo[cb], sc[cb][tb0 + i]);
                }
            };
            __builtin_amdgcn_s_setprio(1);
            scores(std::integral_constant<int, 0>{});
            scores(std::integral_constant<int, 2>{});
            __builtin_amdgcn_s_setprio(0);
            bf16x8 pb[NB][2];
            C.softmax(sc, edge, p0, ks, Q.s, vs, pb);
            const uint32_t va = (uint32_t)(uintptr_t)&vl[stg][128 * ((now >> 4) & 3) + (now & 15)];
            auto vals = [&](auto d0_t) __attribute__((always_inline)) {
                constexpr int d0 = decltype(d0_t)::value;
                u32x4 v[4];
                lds_run<d0 * 256, 256>(va, v);
                if (edge) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t mask = C.v_mask(p0, j);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i][j] &= mask;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bf16x8 f = widen(v[i][2 * h], v[i][2 * h + 1]);
#pragma unroll
                        for (int cb = 0; cb < NB; ++cb) C.o[cb][d0 + i] = mfma16x16x32(f, pb[cb][h], C.o[cb][d0 + i]);
                    }
                }
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
            Q.load(A, nx, t0, A.mw);
            C.begin(nx.s, t0, A.mw, r);
        }
        it = nx;
        --left;
    }
}

// Slot of piece i of an item that share w0 begins.
__device__ __forceinline__ size_t slot_of(int w0, int i) { return 2 * (size_t)(w0 + i) + (i == 0 ? 1 : 0); }

constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / 64;

// Joins np pieces of NC columns, half a wave a piece, 8 requested at a time: lane holds dimensions 4 (lane % 32) .. + 3 of
// num.  piece(i, j): piece i of column j.
template <int NC, class Piece>
__device__ __forceinline__ void join_halves(int np, Piece piece, f32x4 (&num)[NC], float (&den)[NC]) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    float M[NC], wt[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        M[j] = -INFINITY;
        den[j] = 0.f;
        num[j] = f32x4{};
    }
    for (int s0 = 0; s0 < np; s0 += 64) {
        const int k = min(np - s0, 64);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            float m = -INFINITY, l = 0.f;
            if (lane < k) {
                const float* p = piece(s0 + lane, j);
                m = p[D];
                l = p[D + 1];
            }
            const float Mn = fmaxf(M[j], wave_max(m)), f = exp2f(M[j] - Mn);
            wt[j] = exp2f(m - Mn);
            den[j] = den[j] * f + wave_sum(wt[j] * l);
            num[j] *= f;
            M[j] = Mn;
        }
        for (int i = 0; i < k; i += 8) {
            f32x4 v[NC][4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < NC; ++j)       // a piece past the last weighs nothing
                    v[j][u] = *(const f32x4*)(piece(s0 + min(i + 2 * u + half, k - 1), j) + 4 * (lane & 31));
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < NC; ++j) num[j] += __shfl(wt[j], i + 2 * u + half) * v[j][u];
        }
    }
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) num[j][e] += __shfl_xor(num[j][e], 32);
}

// One new row a sequence or a few (an item is a sequence and K/V head): a workgroup a column.  Wave
// v takes pieces v, v + 4, ...: lane i holds the maximum and sum of its i-th, every lane two of the
// 128 dimensions; the waves meet in LDS.
__global__ __launch_bounds__(kJoinThreads) void join_few_kernel(AttnArgs A) {
    __shared__ float num_s[kJoinWaves][D], m_s[kJoinWaves], den_s[kJoinWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int x = blockIdx.x / A.cols, c = blockIdx.x % A.cols, b = x / A.g, kvh = x % A.g, r = A.a / A.g;
    const SeqRows s = seq_rows(A.r, b);
    const int t = c / r;
    if (t >= s.n) return;
    const int w0 = A.cut[x].x, np = A.cut[x].y;
    if (np == 1) return;                       // written by its wave
    const size_t step = (size_t)A.cols * PSTRIDE;
    const float* part = A.part + (size_t)c * PSTRIDE;
    const int mine = (np - wave + kJoinWaves - 1) / kJoinWaves;
    float M = -INFINITY, den = 0.f;
    f32x2 num = {0.f, 0.f};
    for (int s0 = 0; s0 < mine; s0 += 64) {
        const int k = min(mine - s0, 64);
        auto piece = [&](int i) { return part + slot_of(w0, wave + kJoinWaves * (s0 + i)) * step; };
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

// The same where items have few pieces: a wave a column.
__global__ __launch_bounds__(kJoinThreads) void join_short_kernel(AttnArgs A) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = A.a / A.g;
    const int y = blockIdx.x * kJoinWaves + wave;
    if (y >= A.r.B * A.g * A.cols) return;
    const int x = y / A.cols, c = y % A.cols, b = x / A.g, kvh = x % A.g;
    const SeqRows s = seq_rows(A.r, b);
    const int t = c / r;
    if (t >= s.n) return;
    const int w0 = A.cut[x].x, np = A.cut[x].y;
    if (np == 1) return;                       // written by its wave
    const size_t step = (size_t)A.cols * PSTRIDE;
    const float* part = A.part + (size_t)c * PSTRIDE;
    f32x4 num[1];
    float den[1];
    join_halves<1>(np, [&](int i, int) { return part + slot_of(w0, i) * step; }, num, den);
    u32x2 o = {pack2bf(num[0][0] / den[0], num[0][1] / den[0]), pack2bf(num[0][2] / den[0], num[0][3] / den[0])};
    if (t >= s.act) o = u32x2{0, 0};
    if (lane < 32) *(u32x2*)(A.out + ((size_t)(s.row0 + t) * A.a + kvh * r + c % r) * D + 4 * lane) = o;
}

// Many rows: workgroups for each share, which join the item that it begins and does not end; a wave a pair
// of columns, with the pieces of both requested together.
constexpr int kJoinCols = 2 * kJoinWaves;
__global__ __launch_bounds__(kJoinThreads) void join_many_kernel(AttnArgs A) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = A.a / A.g, w0 = blockIdx.x;
    const CutItem it = A.cut_many[w0];
    if (it.np == 0) return;
    const size_t step = (size_t)A.cols * PSTRIDE;
    const int c0 = kJoinCols * blockIdx.y + 2 * wave;
    const int cols = min(A.cols, it.n * r);
    if (c0 >= cols) return;
    float M[2] = {-INFINITY, -INFINITY}, den[2] = {0.f, 0.f};
    f32x2 num[2] = {{0.f, 0.f}, {0.f, 0.f}};
    for (int i0 = 0; i0 < it.np; i0 += 2) {
        f32x2 v[2][2], ml[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // A piece past the last and a column past the item's repeat the last one.
                const float* p = A.part + slot_of(w0, min(i0 + i, it.np - 1)) * step + (size_t)min(c0 + j, cols - 1) * PSTRIDE;
                v[i][j] = *(const f32x2*)(p + 2 * lane);
                ml[i][j] = *(const f32x2*)(p + D);
            }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (i0 + i >= it.np) continue;
                const float Mn = fmaxf(M[j], ml[i][j][0]), f = exp2f(M[j] - Mn), wt = exp2f(ml[i][j][0] - Mn);
                den[j] = den[j] * f + wt * ml[i][j][1];
                num[j][0] = num[j][0] * f + wt * v[i][j][0];
                num[j][1] = num[j][1] * f + wt * v[i][j][1];
                M[j] = Mn;
            }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = c0 + j, t = c / r;
        if (c >= cols) break;
        const uint32_t o = t < it.act ? pack2bf(num[j][0] / den[j], num[j][1] / den[j]) : 0u;
        *(uint32_t*)(A.out + ((size_t)(it.row + t) * A.a + it.head + c % r) * D + 2 * lane) = o;
    }
}

// The same where items have many pieces.
__global__ __launch_bounds__(kJoinThreads) void join_long_kernel(AttnArgs A) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = A.a / A.g, w0 = blockIdx.x;
    const CutItem it = A.cut_many[w0];
    if (it.np == 0) return;
    const int c0 = kJoinCols * blockIdx.y + 2 * wave;
    const int cols = min(A.cols, it.n * r);
    if (c0 >= cols) return;
    const size_t step = (size_t)A.cols * PSTRIDE;
    f32x4 num[2];
    float den[2];
    // A column past the item's repeats the last one.
    join_halves<2>(it.np, [&](int i, int j) { return A.part + slot_of(w0, i) * step + (size_t)min(c0 + j, cols - 1) * PSTRIDE; }, num,
                   den);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = c0 + j, t = c / r;
        if (c >= cols) break;
        u32x2 o = {pack2bf(num[j][0] / den[j], num[j][1] / den[j]), pack2bf(num[j][2] / den[j], num[j][3] / den[j])};
        if (t >= it.act) o = u32x2{0, 0};
        if (lane < 32) *(u32x2*)(A.out + ((size_t)(it.row + t) * A.a + it.head + c % r) * D + 4 * lane) = o;
    }
}

// Shares of the list.  Few: one wave a SIMD (of 1, 1.5, 2 and 3 a SIMD, us: 64 x 32768 positions 738, 743,
// 746, 761; 8 x 64K-128K 287, 290, 292, 299; 16 x 4 rows over 1500-8000 positions 44, 46, 47, 52; 3/4 of a wave
// 739, 289, 45; half a wave 930, 359, 50; requesting two tiles ahead changes none of them).  Many: as many
// workgroups as a CU holds, three with 32 columns a wave (two, without a limit on the registers: prompts of 4 x
// 4096 rows 6 % slower), four with 16.
int few_shares(int simds) { return std::min(simds, kMaxDecodeSplits); }
int many_shares(int simds, int nb) { return std::max(1, (nb == 1 ? 4 : 3) * simds / 4); }

// Up to here a wave takes all columns of an item: 16 sequences over 1500-8000 positions, 32 heads on 8, 8 rows
// each (32 columns) 52 us, on attention_many_kernel 67; 12 rows (48 columns) 76 against 61.
constexpr int kFewCols = 32;
template <int NB>
void launch_few(int nw, int grid, const AttnArgs& A, hipStream_t st) {
    if (nw == 0) hipLaunchKernelGGL((attention_few_kernel<0, NB>), dim3(grid), dim3(64), 0, st, A);
    else if (nw == 1) hipLaunchKernelGGL((attention_few_kernel<1, NB>), dim3(grid), dim3(64), 0, st, A);
    else if (nw == 2) hipLaunchKernelGGL((attention_few_kernel<2, NB>), dim3(grid), dim3(128), 0, st, A);
    else hipLaunchKernelGGL((attention_few_kernel<8, NB>), dim3(grid), dim3(512), 0, st, A);
}
template <int NB>
void launch_many(bool list, int grid, const AttnArgs& A, hipStream_t st) {
    if (list) hipLaunchKernelGGL((attention_many_kernel<true, NB>), dim3(grid), dim3(256), 0, st, A);
    else hipLaunchKernelGGL((attention_many_kernel<false, NB>), dim3(grid), dim3(256), 0, st, A);
}

// Waves that take an item of few columns where a launch without a list and a join is the faster one, else 0.  One
// workgroup an item against the list, 32 heads on 8, in us: 1 sequence of 500 positions 6.5 against 8.4, 1000 8.7
// against 8.7, 2000 13.1 against 9.2; 8 sequences of 1000 9.6 against 11.2, 2000 14.7 against 14.4; 16 of 2000 15.1
// against 19.0, 4000 34 against 33; 64 of 500 14.8 against 19.5, 2000 53 against 59; 100 of 1000 41 against 54.  (Past
// 2048 positions one long sequence among short ones would cost more than there is to gain.)  8, 2 and 1 waves: 32
// sequences of 500 positions 9.5, 9.8 and 12.9; 64 of 1000 31, 29 and 36; 100 of 1000 51, 46 and 41; 16 of 60 4.7,
// 4.6 and 4.1.
int few_waves(int64_t items, int max_pos, int simds) {
    if (max_pos < 2 * TILE) return 1;
    if (max_pos >= std::min<int64_t>(2048, 900 + 17 * items)) return 0;
    return items <= simds / 4 ? 8 : items <= simds / 2 ? 2 : 1;
}

}  // namespace

// Pieces, then what the join reads.
size_t attention_fp8_bytes(int B, int g, int simds) {
    const size_t pieces = (size_t)2 * PSTRIDE * sizeof(float) * std::max(32 * few_shares(simds), 128 * many_shares(simds, 2));
    return pieces + std::max((size_t)B * g * sizeof(int2), (size_t)many_shares(simds, 1) * sizeof(CutItem));
}

hipError_t attention_fp8(const NewRows& r, int a, int g, const uint16_t* q, const uint8_t* kc, const uint8_t* vc,
                         const float* sc, uint16_t* out, void* ws, int simds, hipStream_t st) {
    if (r.B < 1 || r.rows < 1 || r.n_pages < 1 || r.stride < 1 || a % g || a / g > 16) return hipErrorInvalidValue;
    const int heads = a / g;
    // The list counts tiles in 31 bits; where it might not, items run one by one.
    auto listed = [&](int64_t items) { return items * (r.max_pos / TILE + 1) <= INT32_MAX; };
    AttnArgs A{r, q, kc, vc, sc, out, (float*)ws, a, g, 0, 0, 0, nullptr, nullptr, (float)(1.4426950408889634 / sqrt((double)D))};
    hipError_t e;
    if (r.max_new * heads <= kFewCols) {
        A.m = r.max_new;
        A.cols = A.m * heads;
        const int items = r.B * g, nw = listed(items) ? few_waves(items, r.max_pos, simds) : 1;
        if (nw) {
            if (A.cols <= 16) launch_few<1>(nw, items, A, st);
            else launch_few<2>(nw, items, A, st);
            return hipGetLastError();
        }
        const int shares = few_shares(simds);
        A.cut = (int2*)(A.part + (size_t)2 * shares * A.cols * PSTRIDE);
        if (A.cols <= 16) launch_few<1>(0, shares, A, st);
        else launch_few<2>(0, shares, A, st);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        // Few pieces an item, a wave a column: 14 x 4630 positions, 4 rows, 64 heads on 8, 41 us (four waves a column
        // 45).  Many, four waves: 30000 positions, 5 heads on 1 (469 pieces) 17 us (one wave 38); 2 x 5000, 32 on 8
        // (64) 13.3 (15.7).
        if (shares <= 32 * items)
            hipLaunchKernelGGL(join_short_kernel, dim3((items * A.cols + kJoinWaves - 1) / kJoinWaves), dim3(kJoinThreads), 0, st, A);
        else
            hipLaunchKernelGGL(join_few_kernel, dim3(items * A.cols), dim3(kJoinThreads), 0, st, A);
        return hipGetLastError();
    }
    // Rows of a wave: what its 16 (where they hold a quarter of the longest sequence's rows: 14 sequences of 4630
    // positions, 5 rows, 64 heads on 8, 48 us against 56) or 32 columns hold, and no more than that quarter.
    const int nb = 4 * (16 / heads) >= r.max_new ? 1 : 2;
    A.mw = std::min(16 * nb / heads, (r.max_new + 3) / 4);
    A.m = 4 * A.mw;
    A.cols = A.m * heads;
    const int shares = many_shares(simds, nb);
    const int64_t items = (int64_t)g * (r.rows / A.m + r.B), grid = (int64_t)g * r.B * ((r.max_new + A.m - 1) / A.m);
    // Items one by one or the list, in us.  One by one: the tiles of the longest one after the other, a part of all
    // work, and blocks that are none (the grid has as many for every sequence as the longest may have).  The list: all
    // work shared evenly, a second launch, and the pieces' way to memory and back.  Of the tiles some 0.6 of the most
    // that there may be.  Measured, 32 heads on 8, one by one and listed: 1 prompt of 2000 rows 70 and 86, 3 of
    // 395-791 36 and 60, 3 x 333-1001 rows behind 700-5000 positions 163 and 137, 512 rows behind 8000 224 and 103.
    const double n = r.max_pos / TILE + 1, T = 0.6 * items * n;
    const double one = 6 + 1.65 * n + T / 512 + grid / 2000.,
                 list = 12 + T / 256 + (std::min<double>(T, shares) + items) * A.cols * (PSTRIDE * sizeof(float)) / 2.3e6;
    const bool fits = grid < 1 << 24;       // 2^32 threads
    if ((one < list && fits) || !listed(items)) {
        if (!fits) return hipErrorInvalidValue;
        nb == 1 ? launch_many<1>(false, grid, A, st) : launch_many<2>(false, grid, A, st);
        return hipGetLastError();
    }
    A.cut_many = (CutItem*)(A.part + (size_t)2 * shares * A.cols * PSTRIDE);
    nb == 1 ? launch_many<1>(true, shares, A, st) : launch_many<2>(true, shares, A, st);
    if ((e = hipGetLastError()) != hipSuccess || shares == 1) return e;
    // Few items have many pieces each: 7-140 rows behind 4 x 31355 positions 61 us against 77; with two or three pieces
    // an item (700-5000 positions above) 137 against 143 the other way.
    const dim3 join(shares - 1, (A.cols + kJoinCols - 1) / kJoinCols);
    if (4 * items <= shares)
        hipLaunchKernelGGL(join_long_kernel, join, dim3(kJoinThreads), 0, st, A);
    else
        hipLaunchKernelGGL(join_many_kernel, join, dim3(kJoinThreads), 0, st, A);
    return hipGetLastError();
}

}  // namespace kvp
