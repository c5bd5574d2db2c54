// Attention of a call's new rows over a paged cache, whatever its pages hold: the list of tiles, its
// shares, the items of a share, and the join of pieces (device helpers shared by the 8-bit and the bf16 cache's
// kernels).
//
// The rows of a sequence and the r = a / g query heads of a K/V head are the columns of one product; a block of m rows
// makes an item for each K/V head, and an item has a tile for each page (64 positions) that some of its rows sees.  The
// tiles of all items, in the order (sequence, K/V head, block, tile), are one list, which the shares (waves or workgroups)
// cut evenly: an item that begins and ends with one share is written by it, the others leave their pieces (running
// maximum, sum, unnormalised O) to a second kernel, the join.
//
// WIN: a row at position p sees positions [0, p] that lie in its window, above p - window, or below `sinks`.  An item's
// tiles are then the first ones, which hold the positions below `sinks`, and those from the first position on that lies in
// its first row's window; the `gap` tiles between are none of the list's.
#pragma once

#include "fp8_cache.h"

namespace kvp {
namespace {

constexpr int D = kHead, TILE = kPage;
constexpr int PSTRIDE = D + 4;    // O[128], m, l, pad
constexpr float kLazy = 8.0f;     // the running maximum follows once it is 2^8 behind

struct CutItem {
    int np, row, n, act, head, pad[3];     // pieces; first row in the tensors, rows (of them act see something), first head
};

struct ListArgs {
    NewRows r;
    uint16_t* out;
    float* part;       // [2 W][cols][PSTRIDE]: slot 2 w: share w's piece of an item that began before it,
                       // 2 w + 1: of one that begins with it and goes on
    int a, g;
    int m, cols;       // rows of an item, columns that they make
    int mw;            // rows of a wave where several share an item's tiles: m / 4
    // What the join reads: of few columns, for each sequence and K/V head the share that begins it and how many shares
    // have a part; of many, for each share the item that it begins and does not end (np 0: none).
    int2* cut;
    struct CutItem* cut_many;
    int window, sinks; // WIN only: 1 .. 2^30, 0 .. 2^30
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

// Tiles that hold the positions below A.sinks.
__device__ __forceinline__ int sink_tiles(const ListArgs& A) { return (A.sinks + TILE - 1) / TILE; }
// Tiles between those and the first one in the window of a row at position p: behind every later row's window too.
__device__ __forceinline__ int gap_at(const ListArgs& A, int p) {
    return max(p - A.window + 1 - TILE * sink_tiles(A), 0) / TILE;
}
// Tiles of block c of a sequence, and of its first c blocks (without a window); a block without a row that sees anything
// counts one (it writes zeros).
template <bool WIN>
__device__ __forceinline__ int tiles_of(const ListArgs& A, const SeqRows& s, int c) {
    const int last = min((c + 1) * A.m, s.act) - 1;
    if (last < c * A.m) return 1;
    return (s.len + last) / TILE + 1 - (WIN ? gap_at(A, s.len + c * A.m) : 0);
}
__device__ __forceinline__ uint32_t tiles_before(const ListArgs& A, const SeqRows& s, int c) {
    const int m = A.m, full = min(c, s.act / m);            // blocks whose m rows all see something
    uint32_t n = full + floor_sum(full, TILE, m, s.len + m - 1);
    if (c > full) n += tiles_of<false>(A, s, full) + (c - full - 1);
    return n;
}
__device__ __forceinline__ int blocks_of(const SeqRows& s, int m) { return (s.n + m - 1) / m; }
// FEW: every sequence has one block at most.  (With a window there is no other list.)
template <bool FEW, bool WIN>
__device__ __forceinline__ uint32_t seq_tiles(const ListArgs& A, const SeqRows& s) {
    static_assert(FEW || !WIN);
    if (FEW) return s.n ? tiles_of<WIN>(A, s, 0) : 0;
    return tiles_before(A, s, blocks_of(s, A.m));
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
template <bool FEW, bool WIN>
struct Lanes {
    int b0;
    SeqRows s;
    uint32_t n, pre;     // pre: before this lane's sequence
    uint32_t total;      // tiles of the 64
    __device__ __forceinline__ void load(const ListArgs& A, int b0_, uint32_t base) {
        const int lane = threadIdx.x & 63;
        b0 = b0_;
        s = SeqRows{0, 0, 0, 0};
        n = 0;
        if (b0 + lane < A.r.B) {
            s = seq_rows(A.r, b0 + lane);
            n = seq_tiles<FEW, WIN>(A, s);
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
template <bool FEW, bool WIN>
__device__ __forceinline__ uint32_t list_tiles(const ListArgs& A, Lanes<FEW, WIN>& L) {
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
    int gap;             // WIN: see above
    // The tile's place in the sequence: its page.
    template <bool WIN>
    __device__ __forceinline__ int at(const ListArgs& A) const {
        return WIN && t >= sink_tiles(A) ? t + gap : t;
    }
    // Tiles and gap of block c.
    template <bool WIN>
    __device__ __forceinline__ void begin(const ListArgs& A) {
        n = tiles_of<WIN>(A, s, c);
        gap = WIN && c * A.m < s.act ? gap_at(A, s.len + c * A.m) : 0;
    }
};
// The item that holds tile x of the list (x < T).
template <bool FEW, bool WIN>
__device__ __forceinline__ Item find_tile(const ListArgs& A, Lanes<FEW, WIN>& L, uint32_t x) {
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
        uint32_t n0 = tiles_before(A, it.s, c);
        while (c > 0 && n0 > rem) n0 -= tiles_of<WIN>(A, it.s, --c);
        for (; c < cmax; ++c) {
            const uint32_t k = tiles_of<WIN>(A, it.s, c);
            if (n0 + k > rem) break;
            n0 += k;
        }
        it.c = c;
        it.t = rem - n0;
    }
    it.begin<WIN>(A);
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
template <bool FEW, bool WIN>
__device__ __forceinline__ bool take_share(const ListArgs& A, Split* sp, uint32_t* w, uint32_t* left, Item* it) {
    Lanes<FEW, WIN> L;
    const bool bounded = FEW || rows_bounded(A.r);
    *sp = Split(list_tiles<FEW, WIN>(A, L), gridDim.x);
    if (!bounded || blockIdx.x >= sp->W) return false;
    // Shares in one block on one XCD: neighbours read the same K/V head.
    *w = xcd_remap(blockIdx.x, sp->W);
    const uint32_t x = sp->start(*w);
    *left = sp->start(*w + 1) - x;
    *it = find_tile<FEW, WIN>(A, L, x);
    return true;
}
// The item behind `it` in the list; false past the end.
template <bool WIN>
__device__ __forceinline__ bool next_item(const ListArgs& A, Item& it) {
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
    it.begin<WIN>(A);
    return true;
}

// Index of the page of an item's tile, for it.kvh.  A wave keeps 64 entries of a table row, so that one
// dependent load serves 64 tiles.
template <bool WIN>
struct Table {
    int b = -1, c = -1, v = 0;
    __device__ __forceinline__ size_t page(const ListArgs& A, const Item& i) {
        const int t = i.at<WIN>(A);
        if (i.b != b || (t >> 6) != c) {
            b = i.b;
            c = t >> 6;
            const int e = 64 * c + (threadIdx.x & 63);
            v = e < A.r.stride ? A.r.pt[(size_t)i.b * A.r.stride + e] : 0;
        }
        const int pg = min(max(__builtin_amdgcn_readlane(v, t & 63), 0), A.r.n_pages - 1);
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
__global__ __launch_bounds__(kJoinThreads) void join_few_kernel(ListArgs A) {
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
__global__ __launch_bounds__(kJoinThreads) void join_short_kernel(ListArgs A) {
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

}  // namespace
}  // namespace kvp
