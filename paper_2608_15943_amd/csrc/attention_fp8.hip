// Attention of a call's new rows over the 8-bit paged cache: one new token a sequence, a few, or
// a whole prompt; row i of sequence b sits at position len_b + i and sees positions [0, len_b + i].
//
// The rows of a sequence and the r = a / g query heads of a K/V head are the columns of one
// product: column c is head c % r of row c / r, and a wave takes 16 NB of them.  It runs over its
// 64-position tiles once with the running maximum and sum of the softmax, without LDS or barriers:
// K and V go from memory to registers in 16-byte runs, are widened to bf16 there (exactly: e4m3
// has 4 significant bits) and multiplied on v_mfma_f32_16x16x32_bf16.
//
//   S^T = K Q^T  Row rho of score block tb is position 16 (rho / 4) + 4 tb + rho % 4 of the tile, so
//                that lane group grp ends with positions 16 grp .. 16 grp + 15: one scale block, and
//                the run that the second product sums over.  The K scale multiplies a lane's
//                scores, one factor for all of them.
//   O^T += V^T P^T  The V scale multiplies P before it is rounded to bf16 (8 bits).
//
// Work is split over the keys too where there are few columns: piece s of ns of an item takes an
// equal share of its tiles, and a second kernel joins the pieces.
#include <math.h>

#include <algorithm>

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

struct Tile8 {
    u32x4 k[4][2];     // [score block][64-dimension half]
    u32x4 v[8];        // [16-dimension block]
    float ks, vs;      // scales of the lane group's 16 positions
};

struct AttnArgs {
    NewRows r;
    const uint16_t* q;
    const uint8_t* kc;
    const uint8_t* vc;
    const float* sc;
    uint16_t* out;
    float* part;       // [piece][16 NB][PSTRIDE]
    int a, g, ns;
    float scale_log2;
};

// One item: 16 NB columns of one sequence and K/V head.
template <int NB>
struct Item {
    int b, kvh, c0, r;       // first column
    SeqRows s;
    int n;                   // tiles that some column sees
    __device__ __forceinline__ int cols() const { return s.n * r; }
};

template <int NB>
__device__ __forceinline__ bool locate(const AttnArgs& A, int x, Item<NB>* it) {
    const int r = A.a / A.g, C = 16 * NB;
    int first;
    auto blocks = [&](const SeqRows& s) { return (s.n * r + C - 1) / C; };
    if (!find_item(A.r, x / A.g, blocks, &it->b, &it->s, &first)) return false;
    it->kvh = x % A.g;
    it->r = r;
    it->c0 = (x / A.g - first) * C;
    // The last of its rows that lies at a position of the call's reach.
    const int t = min((it->c0 + C - 1) / r, it->s.act - 1);
    it->n = t < it->c0 / r ? 0 : (it->s.len + t) / TILE + 1;
    return true;
}

template <int NB>
__global__ __launch_bounds__(64) void attention_kernel(AttnArgs A) {
    const int lane = threadIdx.x, col = lane & 15, grp = lane >> 4;
    const int piece = blockIdx.x, x = piece / A.ns, sp = piece % A.ns;
    Item<NB> it;
    if (!locate<NB>(A, x, &it)) return;
    const SeqRows& s = it.s;
    const int t_begin = (int)((int64_t)it.n * sp / A.ns), t_end = (int)((int64_t)it.n * (sp + 1) / A.ns);
    if (A.ns > 1 && t_begin == t_end) return;     // the join knows

    // Columns: their row's position (the last they see), -1 where there is none.
    int lim[NB], row[NB], head[NB];
    bool real[NB];
    bf16x8 qf[NB][4];
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) {
        const int c = it.c0 + 16 * cb + col, t = c / it.r;
        real[cb] = c < it.cols();
        head[cb] = it.kvh * it.r + c % it.r;
        row[cb] = s.row0 + (real[cb] ? t : 0);
        lim[cb] = real[cb] && t < s.act ? s.len + t : -1;
        const uint16_t* qrow = A.q + ((size_t)row[cb] * A.a + head[cb]) * D + 16 * grp;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            u32x4 w = u32x4{0, 0, 0, 0};
            if (lim[cb] >= 0) w = *(const u32x4*)(qrow + 64 * (ks >> 1) + 8 * (ks & 1));
            qf[cb][ks] = as_bf16x8(w);
        }
    }
    // Positions that every column sees, and the last that one does.
    const int all = s.len + it.c0 / it.r, last = s.len + min((it.c0 + 16 * NB - 1) / it.r, s.act - 1);
    const bool full = it.c0 + 16 * NB <= s.act * it.r;

    int pc = -1, pgv = 0;
    auto load = [&](int t, Tile8& tl) {
        if ((t >> 6) != pc) {
            pc = t >> 6;
            const int e = 64 * pc + lane;
            pgv = e < A.r.stride ? A.r.pt[(size_t)it.b * A.r.stride + e] : 0;
        }
        const int pg = min(max(__builtin_amdgcn_readlane(pgv, t & 63), 0), A.r.n_pages - 1);
        const size_t at = (size_t)it.kvh * A.r.n_pages + pg;
        const uint8_t* kp = A.kc + at * kPageBytes8 + (16 * (col >> 2) + (col & 3)) * D + 16 * grp;
        const uint8_t* vp = A.vc + at * kPageBytes8 + grp * kBlkBytes + col * kBlk;
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int j = 0; j < 2; ++j) tl.k[tb][j] = *(const u32x4*)(kp + 4 * tb * D + 64 * j);
#pragma unroll
        for (int db = 0; db < 8; ++db) tl.v[db] = *(const u32x4*)(vp + 16 * db * kBlk);
        const float* sp = A.sc + at * 2 * kPageBlks + grp;
        tl.ks = sp[0];
        tl.vs = sp[kPageBlks];
    };

    f32x4 o[NB][8];
    float m_run[NB], l_run[NB];
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) {
        m_run[cb] = kNoScore;
        l_run[cb] = 0.f;
#pragma unroll
        for (int db = 0; db < 8; ++db) o[cb][db] = f32x4{};
    }
    Tile8 cur, nxt;
    if (t_begin < t_end) load(t_begin, cur);
    for (int t = t_begin; t < t_end; ++t) {
        if (t + 1 < t_end) load(t + 1, nxt);
        const int p0 = TILE * t + 16 * grp;         // the lane group's first position
        const bool edge = !full || TILE * t + TILE - 1 > all;
        f32x4 sc[NB][4];
#pragma unroll
        for (int cb = 0; cb < NB; ++cb)
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) sc[cb][tb] = f32x4{};
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const bf16x8 kf = widen(cur.k[tb][ks >> 1][2 * (ks & 1)], cur.k[tb][ks >> 1][2 * (ks & 1) + 1]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) sc[cb][tb] = mfma16x16x32(kf, qf[cb][ks], sc[cb][tb]);
            }
        // Lane (col, grp) holds its column's scores at positions p0 + 4 tb + i.
        const float ks = cur.ks * A.scale_log2;
        float vs = cur.vs;
        bf16x8 pb[NB][2];
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) {
            float mx = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (edge && p0 + 4 * tb + i > lim[cb]) sc[cb][tb][i] = -INFINITY;
                    mx = fmaxf(mx, sc[cb][tb][i]);
                }
            const float mt = pair32_max(pair16_max(mx * ks));
            if (__any(mt > m_run[cb] + kLazy)) {
                const float m_new = fmaxf(m_run[cb], mt);
                const float alpha = __builtin_amdgcn_exp2f(m_run[cb] - m_new);
                m_run[cb] = m_new;
                l_run[cb] *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db) o[cb][db] *= alpha;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(fmaf(sc[cb][2 * e + (i >> 2)][i & 3], ks, -m_run[cb]));
                    // Hidden positions weigh nothing whatever their scale holds (0 * NaN).
                    if (edge && p0 + 8 * e + i > lim[cb]) p[i] = 0.f;
                    l_run[cb] += p[i];
                    p[i] *= vs;
                    if (edge && p0 + 8 * e + i > lim[cb]) p[i] = 0.f;
                }
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = pack2bf(p[2 * i], p[2 * i + 1]);
                pb[cb][e] = as_bf16x8(w);
            }
        }
        // Positions that no column sees carry P = 0, but their codes (never written, perhaps) must
        // be finite: they count as 0.
        const bool tail = TILE * t + TILE - 1 > last;
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            u32x4 v = cur.v[db];
            if (tail) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = last + 1 - (p0 + 4 * e);     // bytes of this word that are seen
                    v[e] = left >= 4 ? v[e] : left <= 0 ? 0u : v[e] & ((1u << (8 * left)) - 1u);
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bf16x8 vf = widen(v[2 * e], v[2 * e + 1]);
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) o[cb][db] = mfma16x16x32(vf, pb[cb][e], o[cb][db]);
            }
        }
        if (t + 1 < t_end) cur = nxt;
    }
    // O^T block db: lane holds dimensions 16 db + 4 grp + 0..3 of its column.
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) {
        const float l = pair32_sum(pair16_sum(l_run[cb]));
        if (!real[cb]) continue;
        if (A.ns == 1) {
            const float inv = lim[cb] < 0 ? 0.f : 1.f / l;
            uint16_t* op = A.out + ((size_t)row[cb] * A.a + head[cb]) * D + 4 * grp;
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                const u32x2 w = {pack2bf(o[cb][db][0] * inv, o[cb][db][1] * inv),
                                 pack2bf(o[cb][db][2] * inv, o[cb][db][3] * inv)};
                *(u32x2*)(op + 16 * db) = w;
            }
        } else {
            float* pr = A.part + ((size_t)piece * 16 * NB + 16 * cb + col) * PSTRIDE;
#pragma unroll
            for (int db = 0; db < 8; ++db) *(f32x4*)(pr + 16 * db + 4 * grp) = o[cb][db];
            if (grp == 0) {
                pr[D] = m_run[cb];
                pr[D + 1] = l;
            }
        }
    }
}

// Joins the pieces of an item, a wave a column; a lane has two of the 128 dimensions.
template <int NB>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs A) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int x = blockIdx.x / (4 * NB), cq = blockIdx.x % (4 * NB);
    Item<NB> it;
    if (!locate<NB>(A, x, &it)) return;
    const int cl = 4 * cq + wave, c = it.c0 + cl;
    if (c >= it.cols()) return;
    const int t = c / it.r;
    uint16_t* op = A.out + ((size_t)(it.s.row0 + t) * A.a + it.kvh * it.r + c % it.r) * D + 2 * lane;
    if (t >= it.s.act) {
        *(uint32_t*)op = 0;
        return;
    }
    const float* pr = A.part + ((size_t)x * A.ns * 16 * NB + cl) * PSTRIDE;
    const size_t step = (size_t)16 * NB * PSTRIDE;
    float M = -INFINITY, den = 0.f;
    f32x2 num = {0.f, 0.f};
    for (int s = 0; s < A.ns; ++s, pr += step) {
        if ((int64_t)it.n * s / A.ns == (int64_t)it.n * (s + 1) / A.ns) continue;
        const float m = pr[D], Mn = fmaxf(M, m), f = exp2f(M - Mn), w = exp2f(m - Mn);
        const f32x2 o = *(const f32x2*)(pr + 2 * lane);
        den = den * f + w * pr[D + 1];
        num[0] = num[0] * f + w * o[0];
        num[1] = num[1] * f + w * o[1];
        M = Mn;
    }
    *(uint32_t*)op = pack2bf(num[0] / den, num[1] / den);
}

constexpr int kColumns = 16;      // columns a wave

// Items the columns of a call can make, and pieces of each: two waves a SIMD if the rows alone do
// not give as many.
int items_of(int B, int rows, int a, int g) { return g * ((int)((int64_t)rows * (a / g) / kColumns) + B); }
int pieces_of(int items, int waves) { return std::max(1, 2 * waves / items); }

}  // namespace

// Pieces are only written apart where there are several an item, at most 2 waves a SIMD in all.
size_t attention_fp8_floats(int waves) { return (size_t)2 * waves * kColumns * PSTRIDE; }

hipError_t attention_fp8(const NewRows& r, int a, int g, const uint16_t* q, const uint8_t* kc, const uint8_t* vc,
                         const float* sc, uint16_t* out, float* part, int waves, hipStream_t st) {
    if (r.B < 1 || r.rows < 1 || r.n_pages < 1 || r.stride < 1 || a / g > 16) return hipErrorInvalidValue;
    // No more pieces than tiles.
    const int items = items_of(r.B, r.rows, a, g), ns = std::min(pieces_of(items, waves), r.max_pos / TILE + 1);
    const AttnArgs A{r, q, kc, vc, sc, out, part, a, g, ns, (float)(1.4426950408889634 / sqrt((double)D))};
    hipLaunchKernelGGL(attention_kernel<1>, dim3(items * ns), dim3(64), 0, st, A);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || ns == 1) return e;
    hipLaunchKernelGGL(join_kernel<1>, dim3(items * 4), dim3(256), 0, st, A);
    return hipGetLastError();
}

}  // namespace kvp
