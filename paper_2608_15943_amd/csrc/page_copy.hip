// Pages copied to others inside the pools of every producer: the pages of sequences that are forked and write on, or that
// a compaction moves.
//
// A page of a producer is, for each K/V head, a run of K and one of V (16 KB each in bf16, 8 KB in 8 bits) and, of the 8-bit
// cache, 32 bytes of scales.  A workgroup copies one run, every load ahead of the first store.
//
// Bound by memory: 1501 pages of 8 K/V heads and 4 producers in bf16 (1.57 GB read and written) 623 us, 5.05 TB/s, a little
// above what a large contiguous copy reaches (4.7); 5 pages in 8 bits 3.3 us, two loads that depend on each other.
#include "common.h"
#include "kernels.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;

struct Args {
    PagePools pools;
    const int32_t* src;
    const int32_t* dst;
    int n, g;
};

// grid: (pair, K/V head, K or V; producer).  WORDS: 16-byte words of a run and thread.
template <int WORDS>
__global__ __launch_bounds__(kThreads) void copy_kernel(Args A) {
    const int z = blockIdx.x & 1, x = blockIdx.x >> 1, h = x % A.g, i = x / A.g, tid = threadIdx.x;
    const PagePools::Pool& P = A.pools.pool[blockIdx.y];
    const int s = A.src[i], d = A.dst[i];
    if (s < 0 || s >= P.n_pages || d < 0 || d >= P.n_pages || s == d) return;
    const size_t hb = (size_t)h * P.n_pages;
    u32x4* base = (u32x4*)(z ? P.v : P.k);
    const u32x4* from = base + (hb + s) * (WORDS * kThreads) + tid;
    u32x4* to = base + (hb + d) * (WORDS * kThreads) + tid;
    u32x4 v[WORDS];
#pragma unroll
    for (int j = 0; j < WORDS; ++j) v[j] = from[j * kThreads];
    u32x4 sc = {0, 0, 0, 0};
    const bool scales = P.sc && tid == 0;       // K's with K's run, V's with V's
    if (scales) sc = *(const u32x4*)(P.sc + ((hb + s) * 2 + z) * 4);
#pragma unroll
    for (int j = 0; j < WORDS; ++j) to[j * kThreads] = v[j];
    if (scales) *(u32x4*)(P.sc + ((hb + d) * 2 + z) * 4) = sc;
}

}  // namespace

hipError_t copy_pages(const PagePools& pools, bool fp8, const int32_t* src, const int32_t* dst, int n, int g, hipStream_t st) {
    if (pools.n < 1 || pools.n > PagePools::kMax || n < 1 || g < 1) return hipErrorInvalidValue;
    // A launch holds less than 2^32 threads.
    const int most = (1 << 23) / (2 * g);
    if (most < 1) return hipErrorInvalidValue;
    for (int i = 0; i < n; i += most) {
        const int c = n - i < most ? n - i : most;
        const Args A{pools, src + i, dst + i, c, g};
        const dim3 grid(2 * c * g, pools.n);
        if (fp8)
            hipLaunchKernelGGL(copy_kernel<2>, grid, dim3(kThreads), 0, st, A);
        else
            hipLaunchKernelGGL(copy_kernel<4>, grid, dim3(kThreads), 0, st, A);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kvp
