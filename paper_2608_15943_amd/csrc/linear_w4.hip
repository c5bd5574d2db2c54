// Products with 4-bit weights: y[m][n] = sum_k x[m][k] (c[n][k] - 8) s[n][k / group], codes c in
// 0..15, scales s in bf16.
//
// Packed weights: for each 16 outputs and 128 inputs one KB, run 16 j + i of 16 bytes holding
// output i: word w inputs 32 w + 8 j + 0..7, the even ones in its low half, the odd ones in its
// high half.  It is what lane (i, j) of a wave multiplies in four v_mfma_f32_16x16x32_bf16, so a
// wave's load is one contiguous KB and nothing is moved between lanes.  The scales follow, for each
// 16 outputs [K / group][16].
//
// A code becomes a bf16 number by placing it in the top four bits of the mantissa of 1.0: 1 + c / 16,
// one shift and one and-or for two codes.  (c - 8) / 16 is 1.5 less, so a second product with the
// constant -1.5 in place of the weights takes 1.5 sum_k x[m][k] off again.  Both run on the matrix
// cores with fp32 sums, which the weights' stream leaves idle; the group's scale multiplies the fp32
// sum of its inputs.
#include "common.h"
#include "kernels.h"

namespace kvp {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// Codes of one word as bf16 numbers 1 + c / 16, in the order of their inputs.
__device__ __forceinline__ bf16x8 widen4(uint32_t w) {
    constexpr uint32_t M = 0x00780078u, One = 0x3F803F80u;
    u32x4 r;
    r[0] = ((w << 3) & M) | One;
    r[1] = ((w >> 1) & M) | One;
    r[2] = ((w >> 5) & M) | One;
    r[3] = ((w >> 9) & M) | One;
    return as_bf16x8(r);
}

__device__ __forceinline__ float bf(uint32_t u) { return __uint_as_float(u << 16); }

// Workgroup: 16 outputs, its waves every kWaves-th 128 inputs; GS groups of scales in 128 inputs.
template <int NMB, int GS>
__global__ __launch_bounds__(kThreads) void linear_kernel(const uint16_t* __restrict__ X, W4Rows W, int M, int N, int K,
                                                          LinearOut out) {
    __shared__ f32x4 red[kWaves][NMB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
    const int m0 = blockIdx.y * 16 * NMB;
    int nb = blockIdx.x, t = 0;
    while (t < 2 && nb >= (W.rows[t] + 15) / 16) nb -= (W.rows[t++] + 15) / 16;
    const size_t nblocks = (W.rows[t] + 15) / 16, KB = K / 128;
    const uint8_t* codes = (const uint8_t*)W.p[t];
    const uint16_t* scales = (const uint16_t*)(codes + nblocks * 8 * K) + (size_t)nb * (KB * GS) * 16 + 4 * kg;
    codes += (size_t)nb * KB * 1024 + 16 * lane;

    f32x4 acc[NMB];
    const uint16_t* xr[NMB];
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb) {
        acc[mb] = f32x4{};
        xr[mb] = X + (size_t)min(m0 + 16 * mb + col, M - 1) * K + 8 * kg;
    }
    const bf16x8 off = as_bf16x8(u32x4{0xBFC0BFC0u, 0xBFC0BFC0u, 0xBFC0BFC0u, 0xBFC0BFC0u});   // -1.5
    for (int kb = wave; kb < (int)KB; kb += kWaves) {
        const u32x4 c = *(const u32x4*)(codes + (size_t)kb * 1024);
#pragma unroll
        for (int gs = 0; gs < GS; ++gs) {
            const u32x2 sw = *(const u32x2*)(scales + (size_t)(kb * GS + gs) * 16);
            const f32x4 sf = {bf(sw[0] & 0xFFFFu), bf(sw[0] >> 16), bf(sw[1] & 0xFFFFu), bf(sw[1] >> 16)};
            f32x4 part[NMB];
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) part[mb] = f32x4{};
#pragma unroll
            for (int w = gs * (4 / GS); w < (gs + 1) * (4 / GS); ++w) {
                const bf16x8 wf = widen4(c[w]);
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb) {
                    const bf16x8 xf = as_bf16x8(*(const u32x4*)(xr[mb] + kb * 128 + 32 * w));
                    part[mb] = mfma16x16x32(wf, xf, part[mb]);
                    part[mb] = mfma16x16x32(off, xf, part[mb]);
                }
            }
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) acc[mb] += sf * part[mb];
        }
    }
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb) red[wave][mb][lane] = acc[mb];
    __syncthreads();
    // Lane (col, kg) of block mb: row 16 mb + col, outputs 4 kg .. + 3.
    for (int i = threadIdx.x; i < 64 * NMB; i += kThreads) {
        const int mb = i >> 6, ln = i & 63, m = m0 + 16 * mb + (ln & 15);
        const int n = blockIdx.x * 16 + 4 * (ln >> 4);
        if (m >= M) continue;
        f32x4 v = red[0][mb][ln];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += red[w][mb][ln];
        v *= 16.f;
        const size_t at = (size_t)m * N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= N) break;
            float y = v[e];
            if (out.res) y += out.res_f32 ? ((const float*)out.res)[at + e] : bf(((const uint16_t*)out.res)[at + e]);
            if (out.y) out.y[at + e] = f2bf(y);
            if (out.yf) out.yf[at + e] = y;
        }
    }
}

// One wave for 16 outputs and 128 inputs: lane (i, j) holds output i, inputs 32 w + 8 j + 0..7.
template <int GS>
__global__ __launch_bounds__(64) void pack_kernel(const uint16_t* __restrict__ W, int N, int K, uint8_t* __restrict__ out) {
    const int lane = threadIdx.x, i = lane & 15, j = lane >> 4;
    const int kb = blockIdx.x, nb = blockIdx.y, n = 16 * nb + i;
    const size_t KB = K / 128;
    float x[4][8];
    uint32_t m[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        u32x4 v = u32x4{0, 0, 0, 0};
        if (n < N) v = *(const u32x4*)(W + (size_t)n * K + 128 * kb + 32 * w + 8 * j);
        m[w] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[w][e] = bf((v[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
            m[w] = max(m[w], __float_as_uint(x[w][e]) & 0x7FFFFFFFu);
        }
        m[w] = max(m[w], (uint32_t)__shfl_xor((int)m[w], 16));
        m[w] = max(m[w], (uint32_t)__shfl_xor((int)m[w], 32));
    }
    uint16_t* scales = (uint16_t*)(out + (size_t)gridDim.y * 8 * K) + (nb * KB + kb) * GS * 16;
    u32x4 c;
#pragma unroll
    for (int gs = 0; gs < GS; ++gs) {
        uint32_t top = 0;
#pragma unroll
        for (int w = gs * (4 / GS); w < (gs + 1) * (4 / GS); ++w) top = max(top, m[w]);
        // The scale that takes the group's largest weight to 7, in bf16; NaN if a weight is not finite.
        uint16_t sb = top >= 0x7F800000u ? 0x7FC0 : f2bf(__uint_as_float(top) / 7.f);
        if (bf(sb) < 0x1p-100f) sb = 0;
        const float s = bf(sb);
        if (j == 0) scales[gs * 16 + i] = sb;
#pragma unroll
        for (int w = gs * (4 / GS); w < (gs + 1) * (4 / GS); ++w) {
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int q = s > 0.f ? (int)fminf(fmaxf(rintf(x[w][e] / s), -8.f), 7.f) + 8 : 8;
                word |= (uint32_t)q << (4 * (e >> 1) + 16 * (e & 1));
            }
            c[w] = word;
        }
    }
    *(u32x4*)(out + ((size_t)nb * KB + kb) * 1024 + 16 * lane) = c;
}

template <int GS>
hipError_t launch(const uint16_t* x, const W4Rows& w, int M, int N, int K, const LinearOut& o, int blocks, hipStream_t st) {
    const int nmb = M > 48 ? 4 : (M + 15) / 16;
    const dim3 grid(blocks, (M + 16 * nmb - 1) / (16 * nmb)), block(kThreads);
    switch (nmb) {
        case 1: hipLaunchKernelGGL((linear_kernel<1, GS>), grid, block, 0, st, x, w, M, N, K, o); break;
        case 2: hipLaunchKernelGGL((linear_kernel<2, GS>), grid, block, 0, st, x, w, M, N, K, o); break;
        case 3: hipLaunchKernelGGL((linear_kernel<3, GS>), grid, block, 0, st, x, w, M, N, K, o); break;
        default: hipLaunchKernelGGL((linear_kernel<4, GS>), grid, block, 0, st, x, w, M, N, K, o); break;
    }
    return hipGetLastError();
}

}  // namespace

size_t w4_bytes(int N, int K, int group) {
    const size_t nb = (N + 15) / 16;
    return nb * 8 * K + nb * 32 * (K / group);
}

bool w4_shape_ok(int K, int group) { return K >= 128 && K % 128 == 0 && (group == 32 || group == 64 || group == 128); }

hipError_t pack_w4(const uint16_t* w, int N, int K, int group, uint8_t* packed, hipStream_t st) {
    if (N < 1 || !w4_shape_ok(K, group)) return hipErrorInvalidValue;
    const dim3 grid(K / 128, (N + 15) / 16), block(64);
    if (grid.y > 65535) return hipErrorInvalidValue;
    if (group == 32)
        hipLaunchKernelGGL(pack_kernel<4>, grid, block, 0, st, w, N, K, packed);
    else if (group == 64)
        hipLaunchKernelGGL(pack_kernel<2>, grid, block, 0, st, w, N, K, packed);
    else
        hipLaunchKernelGGL(pack_kernel<1>, grid, block, 0, st, w, N, K, packed);
    return hipGetLastError();
}

hipError_t linear_w4(const uint16_t* x, const W4Rows& w, int M, int K, int group, const LinearOut& o, hipStream_t st) {
    if (M < 1 || !w4_shape_ok(K, group)) return hipErrorInvalidValue;
    int N = 0, blocks = 0;
    for (int t = 0; t < 3; ++t) {
        // Outputs are counted in blocks of 16 across the parts: only the last may end inside one.
        if (w.rows[t] < 0 || (t < 2 && w.rows[t + 1] && w.rows[t] % 16)) return hipErrorInvalidValue;
        N += w.rows[t];
        blocks += (w.rows[t] + 15) / 16;
    }
    if (!N) return hipErrorInvalidValue;
    if (group == 32) return launch<4>(x, w, M, N, K, o, blocks, st);
    if (group == 64) return launch<2>(x, w, M, N, K, o, blocks, st);
    return launch<1>(x, w, M, N, K, o, blocks, st);
}

}  // namespace kvp
