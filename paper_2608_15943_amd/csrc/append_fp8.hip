// New K and V rows into the 8-bit paged cache, rotated to their positions on the way (RoPE), and
// the call's Q rows rotated beside them.
//
// A workgroup owns the rows that fall into one block of 16 positions of one sequence (a scale's
// extent), for some of the heads: it evaluates the rotation of its at most 16 x 64 angles once,
// in double precision, and its waves take the head vectors (Q, K, V) in turn.  A block that holds
// earlier positions keeps its scale or takes a larger one, and then its earlier codes are
// rescaled.  Only one workgroup ever touches a block and head, so nothing is shared between them
// and the result does not depend on the order in which they run.
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
        if constexpr (N == 2) {
            const uint32_t w = *(const uint32_t*)p;
            x[0] = __uint_as_float(w << 16);
            x[1] = __uint_as_float(w & 0xFFFF0000u);
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

template <class Src>
__global__ __launch_bounds__(kThreads) void append_kernel(Src src, Args A, RopeFreqs th) {
    __shared__ float2 cs[kBlk][kHead / 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int b, first;
    SeqRows s;
    auto blocks = [](const SeqRows& s) { return s.act > 0 ? (s.len + s.act - 1) / kBlk - s.len / kBlk + 1 : 0; };
    if (!find_item(A.r, blockIdx.x, blocks, &b, &s, &first)) return;
    const int blk = s.len / kBlk + (int)blockIdx.x - first, pos0 = blk * kBlk;
    const int lo = max(s.len - pos0, 0), hi = min(s.len + s.act - pos0, kBlk);   // new: lo <= place < hi
    const int row0 = s.row0 + pos0 - s.len;                                       // row of place 0 (if new)
    for (int i = tid; i < (hi - lo) * (kHead / 2); i += kThreads) {
        const int p = lo + i / (kHead / 2), f = i % (kHead / 2);
        double sd, cd;
        sincos((double)(pos0 + p) * th.v[f], &sd, &cd);
        cs[p][f] = make_float2((float)cd, (float)sd);
    }
    __syncthreads();
    const int page = page_of(A.r, b, pos0), pblk = blk % kPageBlks;
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
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
            float* scp = A.sc + (((size_t)h * A.r.n_pages + page) * 2 + 0) * kPageBlks + pblk;
            float sn = e4m3_scale(wave_maxu(m)), f = 1.f;
            if (lo > 0) {
                const float so = *scp;
                if (!(sn > so)) sn = sn == sn ? so : sn;     // keeps the larger; NaN if either is
                f = so / sn;
            }
            const bool bad = sn != sn;
            const float inv = bad ? 0.f : 1.f / sn;
            uint8_t* row = A.kc + ((size_t)h * A.r.n_pages + page) * kPageBytes8 + (pblk * kBlk + p) * kHead + 16 * qd;
            if (fresh || (p < lo && f != 1.f)) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    u32x4 w;
                    if (fresh) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = bad ? 0u : e4m3_pack(x[16 * c + 4 * e] * inv, x[16 * c + 4 * e + 1] * inv,
                                                        x[16 * c + 4 * e + 2] * inv, x[16 * c + 4 * e + 3] * inv);
                    } else {
                        w = *(const u32x4*)(row + 64 * c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = bad ? 0u : e4m3_rescale(w[e], f);
                    }
                    *(u32x4*)(row + 64 * c) = w;
                }
            }
            if (lane == 0) *scp = sn;
        } else {
            // V: a lane holds dimensions 2 lane and 2 lane + 1 of all 16 places, which are two
            // 16-byte runs of the block.
            const int h = hv - A.a - A.g;
            float x[kBlk][2];
            uint32_t m = 0;
#pragma unroll
            for (int p = 0; p < kBlk; ++p) {
                x[p][0] = x[p][1] = 0.f;
                if (p >= lo && p < hi) src.template load<2>(row0 + p, 2, h * kHead + 2 * lane, x[p]);
                m = max(m, max(__float_as_uint(x[p][0]) & 0x7FFFFFFFu, __float_as_uint(x[p][1]) & 0x7FFFFFFFu));
            }
            float* scp = A.sc + (((size_t)h * A.r.n_pages + page) * 2 + 1) * kPageBlks + pblk;
            float sn = e4m3_scale(wave_maxu(m)), f = 1.f;
            if (lo > 0) {
                const float so = *scp;
                if (!(sn > so)) sn = sn == sn ? so : sn;
                f = so / sn;
            }
            const bool bad = sn != sn;
            const float inv = bad ? 0.f : 1.f / sn;
            uint8_t* blkp = A.vc + ((size_t)h * A.r.n_pages + page) * kPageBytes8 + pblk * kBlkBytes + 2 * lane * kBlk;
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                u32x4* run = (u32x4*)(blkp + d * kBlk);
                u32x4 old = u32x4{0, 0, 0, 0}, w;
                if (lo > 0 || hi < kBlk) old = *run;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t nw = bad ? 0u : e4m3_pack(x[4 * e][d] * inv, x[4 * e + 1][d] * inv,
                                                             x[4 * e + 2][d] * inv, x[4 * e + 3][d] * inv);
                    uint32_t ow = old[e];
                    if (f != 1.f) ow = bad ? 0u : e4m3_rescale(ow, f);
                    uint32_t fresh = 0, kept = 0;       // masks of this word's bytes
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int p = 4 * e + i;
                        if (p >= lo && p < hi) fresh |= 0xFFu << (8 * i);
                        if (p < lo) kept |= 0xFFu << (8 * i);
                    }
                    w[e] = (nw & fresh) | (ow & kept) | (old[e] & ~(fresh | kept));
                }
                *run = w;
            }
            if (lane == 0) *scp = sn;
        }
    }
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
    const int per = 4 * kWaves;      // head vectors a workgroup
    // n rows lie in at most n / 16 + 2 blocks.
    const dim3 grid(r.cu ? r.rows / kBlk + 2 * r.B : r.B, (A.vectors + per - 1) / per);
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
