// New K and V rows into the 8-bit paged cache, rotated to their positions on the way (RoPE), and
// the call's Q rows rotated beside them.
//
// Many rows (append_kernel): a workgroup owns the rows that fall into one block of 16 positions of
// one sequence (a scale's extent), for some of the heads: it evaluates the rotation of its at most
// 16 x 64 angles once, in double precision, and its waves take the head vectors (Q, K, V) in turn.
// One row a sequence (append_one_kernel): a wave a head vector.  A block that holds earlier
// positions keeps its scale or takes a larger one, and then its earlier codes are rescaled.  Only
// one wave ever touches a block and head, so nothing is shared between waves and the result does
// not depend on the order in which they run.
//
// Bound by memory: prompts of 4 x 4096 rows (16 query heads, 8 K/V heads, 235 MB) 57 us, 4.1 TB/s; 2568 rows in
// 7 chunks (64, 8; 100 MB) 26.9 us; one row of each of 64 sequences 4.2 us, the latency of three loads that
// depend on each other (length, page, scale).
#include "fp8_cache.h"

namespace kvp {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Largest of a wave's words (unsigned).
__device__ __forceinline__ uint32_t wave_maxu(uint32_t v) {
    auto step = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    v = step(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
    v = step(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = step(r[0], r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return step(q[0], q[1]);
}

// Turns of a position at frequency i, to some 2^-61 of them: the host's factors have 64 bits, the products here keep
// them.  At the farthest position, 2^30, that is 2^-33 of a turn, below half a step of the cosine in fp32.
struct Turns {
    double hi, lo;
    __device__ __forceinline__ Turns(const RopeFreqs& th, int i) : hi(th.hi[0]), lo(th.lo[0]) {
#pragma unroll
        for (int j = 0; j < 6; ++j) {
            const bool on = i >> j & 1;
            const double fh = on ? th.hi[1 + j] : 1.0, fl = on ? th.lo[1 + j] : 0.0;
            const double p = hi * fh, e = fma(hi, fh, -p) + (hi * fl + lo * fh);
            hi = p + e;
            lo = e - (hi - p);
        }
    }
};

// Cosine and sine of pos turns * 2 pi, turns = hi + lo (double each): the product's whole turns go exactly, and
// the series of the rest, at most an eighth of a turn, is off by less than 2^-50.  (The library's sincos takes
// any double and most of the time of a call for few rows.)
__device__ __forceinline__ float2 rotation(int pos, const Turns& turns) {
    const double p = pos, t = p * turns.hi, e = fma(p, turns.hi, -t) + p * turns.lo;
    const double k = rint(4.0 * t);                       // quarter turns
    const double x = (fma(-0.25, k, t) + e) * 6.283185307179586, z = x * x;
    // sum of (-z)^n / (2 n + 1)! and / (2 n)!
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = fma(s, z, 1.0 / 6227020800.0);
    s = fma(s, z, -1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, -1.0 / 5040.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, -1.0 / 6.0);
    s = x * fma(s, z, 1.0);
    c = fma(c, z, -1.0 / 87178291200.0);
    c = fma(c, z, 1.0 / 479001600.0);
    c = fma(c, z, -1.0 / 3628800.0);
    c = fma(c, z, 1.0 / 40320.0);
    c = fma(c, z, -1.0 / 720.0);
    c = fma(c, z, 1.0 / 24.0);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const int q = (int)(long long)k & 3;
    const float cf = (float)(q & 1 ? s : c), sf = (float)(q & 1 ? c : s);
    return make_float2(q == 1 || q == 2 ? -cf : cf, q >= 2 ? -sf : sf);
}

// Rotates the pairs (x1[i], x2[i]); each product and sum rounded by itself.
__device__ __forceinline__ void rotate(float& x1, float& x2, float2 cs) {
#pragma clang fp contract(off)
    const float a = x1 * cs.x - x2 * cs.y, b = x2 * cs.x + x1 * cs.y;
    x1 = a;
    x2 = b;
}

// Head vectors of a row, n consecutive values from a column on, in fp32.
struct Bf16Src {
    const uint16_t *q, *k, *v;
    int ldq, ldkv;
    template <int N>
    __device__ __forceinline__ void load(int row, int z, int col, float* x) const {
        const uint16_t* p = z == 0 ? q + (size_t)row * ldq + col : (z == 1 ? k : v) + (size_t)row * ldkv + col;
        if constexpr (N == 1) {
            x[0] = __uint_as_float((uint32_t)p[0] << 16);
        } else {
#pragma unroll
            for (int c = 0; c < N / 8; ++c) {
                const u32x4 w = *(const u32x4*)(p + 8 * c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[8 * c + 2 * e] = __uint_as_float(w[e] << 16);
                    x[8 * c + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
                }
            }
        }
    }
};

// The sum of a projection's planes, in order.
struct PlaneSrc {
    const float* part;
    int nsplit, N, nq, nkv;
    size_t plane;
    template <int N_>
    __device__ __forceinline__ void load(int row, int z, int col, float* x) const {
        const float* p = part + (size_t)row * N + (z == 0 ? 0 : z == 1 ? nq : nq + nkv) + col;
#pragma unroll
        for (int i = 0; i < N_; ++i) x[i] = p[i];
        for (int s = 1; s < nsplit; ++s) {
            p += plane;
#pragma unroll
            for (int i = 0; i < N_; ++i) x[i] += p[i];
        }
    }
};

struct Args {
    NewRows r;
    int a, g;
    uint16_t* q_out;
    uint8_t* kc;
    uint8_t* vc;
    float* sc;
    int vectors;       // head vectors a row: a (if Q is given), then 2 g (if K and V are)
    int first;         // 0: from the first Q vector, a: from the first K vector
};

// The scale of a block whose new values reach m (float bits) and whose earlier ones have scale old (kept: there
// are any): the new scale, and what the earlier codes are multiplied by.
struct NewScale {
    float s, f, inv;
    bool bad;
    __device__ __forceinline__ NewScale(uint32_t m, bool kept, float old) {
        s = e4m3_scale(m);
        f = 1.f;
        if (kept) {
            if (!(s > old)) s = s == s ? old : s;      // the larger; NaN if either is
            f = old / s;
        }
        bad = s != s;
        inv = bad ? 0.f : 1.f / s;
    }
};

// Many rows: workgroup = the new rows of one block of 16 positions, for some of the head vectors.
template <class Src>
__global__ __launch_bounds__(kThreads) void append_kernel(Src src, Args A, RopeFreqs th) {
    __shared__ float2 cs[kBlk][kHead / 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int b, first;
    SeqRows s;
    auto blocks = [](const SeqRows& s) { return s.act > 0 ? (s.len + s.act - 1) / kBlk - s.len / kBlk + 1 : 0; };
    if (!find_item(A.r, blockIdx.x, blocks, &b, &s, &first)) return;
    const int blk = s.len / kBlk + (int)blockIdx.x - first, pos0 = blk * kBlk;
    const int lo = max(s.len - pos0, 0), hi = min(s.len + s.act - pos0, kBlk);   // new: lo <= place < hi
    const int row0 = s.row0 + pos0 - s.len;                                       // row of place 0 (if new)
    const int page = page_of(A.r, b, pos0), pblk = blk % kPageBlks;
    const Turns turns(th, tid % (kHead / 2));       // kThreads is a multiple of that
    for (int i = tid; i < (hi - lo) * (kHead / 2); i += kThreads) {
        const int p = lo + i / (kHead / 2);
        cs[p][i % (kHead / 2)] = rotation(pos0 + p, turns);
    }
    __syncthreads();
    for (int hv = A.first + blockIdx.y * kWaves + wave; hv < A.first + A.vectors; hv += gridDim.y * kWaves) {
        if (hv < A.a + A.g) {
            // Q and K: lane (place, quarter) holds dimensions 16 quarter .. + 15 and the same of
            // the second half.
            const int p = lane >> 2, qd = lane & 3;
            const bool fresh = p >= lo && p < hi, isq = hv < A.a;
            const int h = isq ? hv : hv - A.a;
            float x[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = 0.f;
            if (fresh) {
                src.template load<16>(row0 + p, isq ? 0 : 1, h * kHead + 16 * qd, x);
                src.template load<16>(row0 + p, isq ? 0 : 1, h * kHead + 64 + 16 * qd, x + 16);
#pragma unroll
                for (int i = 0; i < 16; ++i) rotate(x[i], x[16 + i], cs[p][16 * qd + i]);
            }
            if (isq) {
                if (fresh) {
                    uint16_t* o = A.q_out + ((size_t)(row0 + p) * A.a + h) * kHead + 16 * qd;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        u32x4 w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = pack2bf(x[8 * c + 2 * e], x[8 * c + 2 * e + 1]);
                        *(u32x4*)(o + 64 * (c >> 1) + 8 * (c & 1)) = w;
                    }
                }
                continue;
            }
            float* scp = A.sc + ((size_t)h * A.r.n_pages + page) * 2 * kPageBlks + pblk;
            const float old = lo > 0 ? *scp : 0.f;
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
            const NewScale n(wave_maxu(m), lo > 0, old);
            uint8_t* row = A.kc + ((size_t)h * A.r.n_pages + page) * kPageBytes8 + (pblk * kBlk + p) * kHead + 16 * qd;
            if (fresh || (p < lo && n.f != 1.f)) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    u32x4 w;
                    if (fresh) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = n.bad ? 0u : e4m3_pack(x[16 * c + 4 * e] * n.inv, x[16 * c + 4 * e + 1] * n.inv,
                                                          x[16 * c + 4 * e + 2] * n.inv, x[16 * c + 4 * e + 3] * n.inv);
                    } else {
                        w = *(const u32x4*)(row + 64 * c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = n.bad ? 0u : e4m3_rescale(w[e], n.f);
                    }
                    *(u32x4*)(row + 64 * c) = w;
                }
            }
            if (lane == 0) *scp = n.s;
        } else {
            // V: lane (grp, c) holds dimensions 8 c .. 8 c + 7 of places 4 grp .. 4 grp + 3, whose codes are word
            // grp of the dimensions' 16-byte runs; lanes of the four groups exchange words until each has two
            // whole runs, of dimensions 8 c + grp and 8 c + 4 + grp.
            const int h = hv - A.a - A.g, grp = lane >> 4, c = lane & 15;
            float x[4][8];
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int p = 4 * grp + j;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = 0.f;
                if (p >= lo && p < hi) src.template load<8>(row0 + p, 2, h * kHead + 8 * c, x[j]);
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[j][e]) & 0x7FFFFFFFu);
            }
            float* scp = A.sc + ((size_t)h * A.r.n_pages + page) * 2 * kPageBlks + kPageBlks + pblk;
            const float old = lo > 0 ? *scp : 0.f;
            const NewScale n(wave_maxu(m), lo > 0, old);
            uint8_t* blkp = A.vc + ((size_t)h * A.r.n_pages + page) * kPageBytes8 + pblk * kBlkBytes;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int d = 4 * q + e;
                    w[e] = n.bad ? 0u : e4m3_pack(x[0][d] * n.inv, x[1][d] * n.inv, x[2][d] * n.inv, x[3][d] * n.inv);
                }
                const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const auto b2 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                const auto r0 = __builtin_amdgcn_permlane16_swap(a[0], b2[0], false, false);
                const auto r1 = __builtin_amdgcn_permlane16_swap(a[1], b2[1], false, false);
                u32x4 run = {r0[0], r0[1], r1[0], r1[1]};
                u32x4* dst = (u32x4*)(blkp + (8 * c + 4 * q + grp) * kBlk);
                if (lo > 0 || hi < kBlk) {
                    const u32x4 was = *dst;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t kept = 0, fresh = 0;       // masks of this word's bytes
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int p = 4 * e + i;
                            if (p < lo) kept |= 0xFFu << (8 * i);
                            if (p >= lo && p < hi) fresh |= 0xFFu << (8 * i);
                        }
                        uint32_t o = was[e];
                        if (n.f != 1.f) o = (n.bad ? 0u : e4m3_rescale(o, n.f) & kept) | (o & ~kept);
                        run[e] = (run[e] & fresh) | (o & ~fresh);
                    }
                }
                *dst = run;
            }
            if (lane == 0) *scp = n.s;
        }
    }
}

// One row a sequence at most: a wave a head vector of a row, lane i dimensions i and i + 64; everything that does
// not depend on the position is requested ahead of it.
template <class Src>
__global__ __launch_bounds__(kThreads) void append_one_kernel(Src src, Args A, RopeFreqs th) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int groups = (A.vectors + kWaves - 1) / kWaves;
    const int b = blockIdx.x / groups, hv = A.first + blockIdx.x % groups * kWaves + wave;
    if (hv >= A.first + A.vectors) return;
    const SeqRows s = seq_rows(A.r, b);
    if (s.act < 1) return;
    const int z = hv < A.a ? 0 : hv < A.a + A.g ? 1 : 2, h = z == 0 ? hv : z == 1 ? hv - A.a : hv - A.a - A.g;
    float x1, x2;
    src.template load<1>(s.row0, z, h * kHead + lane, &x1);
    src.template load<1>(s.row0, z, h * kHead + 64 + lane, &x2);
    const Turns turns(th, lane);
    const int pos = s.len, page = page_of(A.r, b, pos), pblk = pos / kBlk % kPageBlks, p = pos % kBlk;
    const size_t at = (size_t)h * A.r.n_pages + page;
    float* scp = A.sc + at * 2 * kPageBlks + (z == 2 ? kPageBlks : 0) + pblk;
    const float old = z && p ? *scp : 0.f;
    if (z < 2) rotate(x1, x2, rotation(pos, turns));
    if (z == 0) {
        uint16_t* o = A.q_out + ((size_t)s.row0 * A.a + h) * kHead + lane;
        o[0] = f2bf(x1);
        o[64] = f2bf(x2);
        return;
    }
    const NewScale n(wave_maxu(max(__float_as_uint(x1) & 0x7FFFFFFFu, __float_as_uint(x2) & 0x7FFFFFFFu)), p > 0, old);
    const uint32_t c = n.bad ? 0u : e4m3_pack(x1 * n.inv, x2 * n.inv, 0.f, 0.f);
    if (z == 1) {
        uint8_t* blkp = A.kc + at * kPageBytes8 + pblk * kBlkBytes;
        if (n.f != 1.f)        // the block's earlier rows, 16 bytes a lane
            for (int i = lane; i < 8 * p; i += 64) {
                u32x4 w = ((u32x4*)blkp)[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = n.bad ? 0u : e4m3_rescale(w[e], n.f);
                ((u32x4*)blkp)[i] = w;
            }
        blkp[p * kHead + lane] = (uint8_t)c;
        blkp[p * kHead + 64 + lane] = (uint8_t)(c >> 8);
    } else {
        uint8_t* blkp = A.vc + at * kPageBytes8 + pblk * kBlkBytes;
        if (n.f != 1.f) {      // the earlier places of the lane's two runs
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                u32x4* run = (u32x4*)(blkp + (lane + 64 * d) * kBlk);
                u32x4 w = *run;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = p - 4 * e;
                    const uint32_t kept = k >= 4 ? 0xFFFFFFFFu : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
                    w[e] = (n.bad ? 0u : e4m3_rescale(w[e], n.f) & kept) | (w[e] & ~kept);
                }
                *run = w;
            }
        }
        blkp[lane * kBlk + p] = (uint8_t)c;
        blkp[(lane + 64) * kBlk + p] = (uint8_t)(c >> 8);
    }
    if (lane == 0) *scp = n.s;
}

// Row x of no sequence: before the first, behind the last, or past max_new of its own.
__global__ __launch_bounds__(256) void clear_kernel(NewRows r, int n, uint16_t* x) {
    const int row = blockIdx.x;
    bool mine = false;
    for (int b = threadIdx.x; b < r.B; b += 256) {
        const SeqRows s = seq_rows(r, b);
        mine |= row >= s.row0 && row < s.row0 + s.n;
    }
    if (__syncthreads_or(mine)) return;
    for (int i = 8 * threadIdx.x; i < n; i += 8 * 256) *(u32x4*)(x + (size_t)row * n + i) = u32x4{0, 0, 0, 0};
}

template <class Src>
hipError_t launch(const Src& src, const Args& A, const RopeFreqs& th, hipStream_t st) {
    const NewRows& r = A.r;
    if (r.B < 1 || r.rows < 1 || r.n_pages < 1 || r.stride < 1 || A.vectors < 1) return hipErrorInvalidValue;
    if (r.max_new == 1) {
        const dim3 grid((A.vectors + kWaves - 1) / kWaves * r.B);
        hipLaunchKernelGGL(append_one_kernel<Src>, grid, dim3(kThreads), 0, st, src, A, th);
        return hipGetLastError();
    }
    const int per = 2 * kWaves;      // head vectors a workgroup
    // n rows lie in at most n / 16 + 2 blocks.
    const dim3 grid(r.rows / kBlk + 2 * r.B, (A.vectors + per - 1) / per);
    hipLaunchKernelGGL(append_kernel<Src>, grid, dim3(kThreads), 0, st, src, A, th);
    return hipGetLastError();
}

}  // namespace

hipError_t append_fp8(const NewRows& r, int a, int g, const uint16_t* q, const uint16_t* k, const uint16_t* v, int ldq,
                      int ldkv, const RopeFreqs& th, uint16_t* q_out, uint8_t* kc, uint8_t* vc, float* sc, hipStream_t st) {
    return launch(Bf16Src{q, k, v, ldq, ldkv}, Args{r, a, g, q_out, kc, vc, sc, (q ? a : 0) + (k ? 2 * g : 0), q ? 0 : a}, th,
                  st);
}

hipError_t append_fp8_planes(const NewRows& r, int a, int g, const float* part, int nsplit, int N, bool producer,
                             const RopeFreqs& th, uint16_t* q_out, uint8_t* kc, uint8_t* vc, float* sc, hipStream_t st) {
    if (nsplit < 1 || N != (a + (producer ? 2 * g : 0)) * kHead) return hipErrorInvalidValue;
    return launch(PlaneSrc{part, nsplit, N, a * kHead, g * kHead, (size_t)r.rows * N},
                  Args{r, a, g, q_out, kc, vc, sc, a + (producer ? 2 * g : 0), 0}, th, st);
}

hipError_t clear_unowned(const NewRows& r, int n, uint16_t* x, hipStream_t st) {
    if (r.rows < 1 || n < 8 || n % 8) return hipErrorInvalidValue;
    hipLaunchKernelGGL(clear_kernel, dim3(r.rows), dim3(256), 0, st, r, n, x);
    return hipGetLastError();
}

}  // namespace kvp
