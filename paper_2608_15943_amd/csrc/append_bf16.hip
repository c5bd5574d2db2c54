// New K and V rows into the paged bf16 cache, rotated to their positions on the way (RoPE), and the call's Q rows rotated
// beside them.
//
// Pages hold 64 positions: K [64][128], V [128][64], the positions of one dimension side by side.  Many rows
// (append_rows_kernel): a workgroup owns the rows that fall into half a page of one sequence, for some of the head vectors
// (Q, K, V): it evaluates the rotation of its at most 32 x 64 angles once, in double precision.  V is turned in registers: a lane
// takes 8 dimensions of 8 positions, whose words it deals out again as 16-byte runs of positions.  One row a sequence
// (append_row_kernel): a wave a head vector.  Only positions of the call's rows that have a page are written, each once.
//
// Bound by memory: 2568 rows in 7 chunks (64 query heads, 8 K/V heads; 105 MB) 26.7 us, 3.9 TB/s (a call from the host 30; 41
// with workgroups of 64 positions and 8 vectors, 31 with 32 and 8 or 16); prompts of 4 x 4096 rows (16, 8; 268 MB) 68 us by such
// calls, 4.0 TB/s (67, 75); one row of each of 8 sequences 3.2 us, the latency of three loads that depend on each other (length,
// page, row).
#include "rope_rows.h"

namespace kvp {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct Args {
    NewRows r;
    int a, g;
    uint16_t* q_out;
    uint16_t* kc;
    uint16_t* vc;
    int vectors;       // head vectors a row: a (if Q is given), then 2 g (if K and V are)
    int first;         // 0: from the first Q vector, a: from the first K vector
};

// Many rows: workgroup = the new rows of kPart positions of one page, for kWaves of the head vectors, one a wave, whose rows
// are requested ahead of the angles.
constexpr int kPart = 32;
template <class Src>
__global__ __launch_bounds__(kThreads) void append_rows_kernel(Src src, Args A, RopeFreqs th) {
    __shared__ float2 cs[kPart][kHead / 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int b, first;
    SeqRows s;
    auto parts = [](const SeqRows& s) { return s.act > 0 ? (s.len + s.act - 1) / kPart - s.len / kPart + 1 : 0; };
    if (!find_item(A.r, blockIdx.x, parts, &b, &s, &first)) return;
    const int pos0 = (s.len / kPart + (int)blockIdx.x - first) * kPart;
    const int lo = max(s.len - pos0, 0), hi = min(s.len + s.act - pos0, kPart);   // new: lo <= place < hi
    const int row0 = s.row0 + pos0 - s.len;                                       // row of place 0 (if new)
    const int hv0 = A.first + blockIdx.y * kWaves, hv = hv0 + wave;
    const int z = hv < A.a ? 0 : hv < A.a + A.g ? 1 : 2, h = z == 0 ? hv : z == 1 ? hv - A.a : hv - A.a - A.g;
    // Q and K: lane (place, c) holds dimensions 8 c .. + 7 (even i) and the same of the second half, 8 (i / 2) places further.
    // V: lane (grp, c) holds dimensions 8 c .. + 7 of places 8 grp + i.
    typename Src::Raw x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int p = z == 2 ? 8 * (lane >> 4) + i : 8 * (i >> 1) + (lane >> 3);
        const int d = z == 2 ? 8 * (lane & 15) : 8 * (lane & 7) + 64 * (i & 1);
        x[i] = typename Src::Raw{};
        if (hv < A.first + A.vectors && p >= lo && p < hi) x[i] = src.raw8(row0 + p, z, h * kHead + d);
    }
    const int page = page_of(A.r, b, pos0), at = pos0 % kPage;
    if (hv0 < A.a + A.g) {
        const Turns turns(th, tid % (kHead / 2));       // kThreads is a multiple of that
        for (int i = tid; i < (hi - lo) * (kHead / 2); i += kThreads) {
            const int p = lo + i / (kHead / 2);
            cs[p][i % (kHead / 2)] = rotation(pos0 + p, turns);
        }
    }
    __syncthreads();
    if (hv >= A.first + A.vectors || (z && page < 0)) return;
    if (z < 2) {
        const int c = lane & 7;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = 8 * i + (lane >> 3);
            if (p < lo || p >= hi) continue;
            float y[16];
            Src::widen(x[2 * i], y);
            Src::widen(x[2 * i + 1], y + 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) rotate(y[e], y[8 + e], cs[p][8 * c + e]);
            uint16_t* o = z == 0 ? A.q_out + ((size_t)(row0 + p) * A.a + h) * kHead + 8 * c
                                 : A.kc + (((size_t)h * A.r.n_pages + page) * kPage + at + p) * kHead + 8 * c;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2bf(y[8 * j + 2 * e], y[8 * j + 2 * e + 1]);
                *(u32x4*)(o + 64 * j) = w;
            }
        }
        return;
    }
    const int c = lane & 15, p0 = 8 * (lane >> 4);
    u32x4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Src::bits(x[i]);
    uint16_t* dst = A.vc + (((size_t)h * A.r.n_pages + page) * kHead + 8 * c) * kPage + at + p0;
    const bool full = p0 >= lo && p0 + 8 <= hi;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        u32x4 run;
#pragma unroll
        for (int j = 0; j < 4; ++j)      // dimension e of two positions
            run[j] = __builtin_amdgcn_perm(v[2 * j + 1][e >> 1], v[2 * j][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
        if (full) {
            *(u32x4*)(dst + e * kPage) = run;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (p0 + j >= lo && p0 + j < hi) dst[e * kPage + j] = (uint16_t)(run[j >> 1] >> (16 * (j & 1)));
        }
    }
}

// One row a sequence at most: a wave a head vector of a row, lane i dimensions i and i + 64; everything that does
// not depend on the position is requested ahead of it.
template <class Src>
__global__ __launch_bounds__(kThreads) void append_row_kernel(Src src, Args A, RopeFreqs th) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int groups = (A.vectors + kWaves - 1) / kWaves;
    const int b = blockIdx.x / groups, hv = A.first + blockIdx.x % groups * kWaves + wave;
    if (hv >= A.first + A.vectors) return;
    const SeqRows s = seq_rows(A.r, b);
    if (s.act < 1) return;
    const int z = hv < A.a ? 0 : hv < A.a + A.g ? 1 : 2, h = z == 0 ? hv : z == 1 ? hv - A.a : hv - A.a - A.g;
    float x1, x2;
    uint16_t y1, y2;
    if (z == 2) {
        y1 = src.v1(s.row0, h * kHead + lane);
        y2 = src.v1(s.row0, h * kHead + 64 + lane);
    } else {
        src.template load<1>(s.row0, z, h * kHead + lane, &x1);
        src.template load<1>(s.row0, z, h * kHead + 64 + lane, &x2);
    }
    const Turns turns(th, lane);
    const int pos = s.len, p = pos % kPage;
    const int page = page_of(A.r, b, pos);
    const size_t at = (size_t)h * A.r.n_pages + max(page, 0);
    if (z < 2) {
        rotate(x1, x2, rotation(pos, turns));
        y1 = f2bf(x1);
        y2 = f2bf(x2);
    }
    if (z && page < 0) return;
    uint16_t* o = z == 0   ? A.q_out + ((size_t)s.row0 * A.a + h) * kHead + lane
                  : z == 1 ? A.kc + (at * kPage + p) * kHead + lane
                           : A.vc + (at * kHead + lane) * kPage + p;
    o[0] = y1;
    o[z == 2 ? 64 * kPage : 64] = y2;
}

template <class Src>
hipError_t launch(const Src& src, const Args& A, const RopeFreqs& th, hipStream_t st) {
    const NewRows& r = A.r;
    if (r.B < 1 || r.rows < 1 || r.n_pages < 1 || r.stride < 1 || A.vectors < 1) return hipErrorInvalidValue;
    if (r.max_new == 1) {
        const dim3 grid((A.vectors + kWaves - 1) / kWaves * r.B);
        hipLaunchKernelGGL(append_row_kernel<Src>, grid, dim3(kThreads), 0, st, src, A, th);
        return hipGetLastError();
    }
    // n rows lie in at most n / 32 + 2 parts of 32 positions.
    const dim3 grid(r.rows / kPart + 2 * r.B, (A.vectors + kWaves - 1) / kWaves);
    hipLaunchKernelGGL(append_rows_kernel<Src>, grid, dim3(kThreads), 0, st, src, A, th);
    return hipGetLastError();
}

}  // namespace

hipError_t append_bf16(const NewRows& r, int a, int g, const uint16_t* q, const uint16_t* k, const uint16_t* v, int ldq,
                       int ldkv, const RopeFreqs& th, uint16_t* q_out, uint16_t* kc, uint16_t* vc, hipStream_t st) {
    return launch(Bf16Src{q, k, v, ldq, ldkv}, Args{r, a, g, q_out, kc, vc, (q ? a : 0) + (k ? 2 * g : 0), q ? 0 : a}, th, st);
}

hipError_t append_bf16_planes(const NewRows& r, int a, int g, const float* part, int nsplit, int N, bool producer,
                              const RopeFreqs& th, uint16_t* q_out, uint16_t* kc, uint16_t* vc, hipStream_t st) {
    if (nsplit < 1 || N != (a + (producer ? 2 * g : 0)) * kHead) return hipErrorInvalidValue;
    return launch(PlaneSrc{part, nsplit, N, a * kHead, g * kHead, (size_t)r.rows * N},
                  Args{r, a, g, q_out, kc, vc, a + (producer ? 2 * g : 0), 0}, th, st);
}

}  // namespace kvp
