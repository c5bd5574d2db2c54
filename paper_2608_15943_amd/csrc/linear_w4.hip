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
// cores with fp32 sums; the group's scale multiplies the fp32 sum of its inputs.
//
// Bound: few rows by reading the weights, in the time that a launch with cold weights allows (1 row, 6144 x 4096,
// 13 MB: 5.5 us, a bare read of as much 3.2; 14000 x 11008, 80 MB: 15.4 us, a bare read 12.5); more rows also by what
// every CU reads of x (16 rows, 8192 x 8192: 9.4 us, 36 MB of weights 6.6), and 33 to 64 by waiting for it: LDS holds
// one stage, so that the products stand still while the next comes (64 rows 19.6 us).  Each further 64 rows read and
// widen the weights again (128 rows 29 us, 4096 795).
#include "common.h"
#include "kernels.h"

namespace kvp {
namespace {

// Codes of one word as bf16 numbers 1 + c / 16, in the order of their inputs.  mask and one (0x00780078,
// 0x3F803F80) come in registers: with literals the and-or is two instructions.
__device__ __forceinline__ bf16x8 widen4(uint32_t w, uint32_t mask, uint32_t one) {
    u32x4 r;
    r[0] = ((w << 3) & mask) | one;
    r[1] = ((w >> 1) & mask) | one;
    r[2] = ((w >> 5) & mask) | one;
    r[3] = ((w >> 9) & mask) | one;
    return as_bf16x8(r);
}

__device__ __forceinline__ float bf(uint32_t u) { return __uint_as_float(u << 16); }

constexpr int NW = 8;      // waves a workgroup

typedef __attribute__((address_space(1))) void gvoid_t;
typedef __attribute__((address_space(3))) void lvoid_t;

// 16-byte LDS reads at a[0..3] + OFF and their wait: written by hand, since the compiler would first wait for the
// loads that go into the other stage.
template <int OFF>
__device__ __forceinline__ void lds_four(const uint32_t (&a)[4], u32x4 (&f)[4]) {
    asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\tds_read_b128 %2, %6 offset:%8\n\t"
                 "ds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "i"(OFF)
                 : "memory");
}

// Workgroup: 16 NT outputs and 16 NMB rows, of them at most ROWS of x; its NW waves take every NW-th 128 inputs.  A
// wave's x goes through a part of LDS of its own, in whole lines of memory: fragments read from memory would touch
// 16 half lines each, which bounded everything from 4 rows on (64 rows, 6144 x 4096: 19 us).  ST 2: the next 128
// inputs are under way during the products (8192 x 8192, 16 rows, 10.0 to 9.4 us); of 64 rows LDS holds one stage.
// GS: groups of scales in 128 inputs.
template <int NMB, int ROWS, int NT, int ST, int GS>
__global__ __launch_bounds__(64 * NW, NW / 4) void linear_kernel(const uint16_t* __restrict__ X, W4Rows W, int M, int N,
                                                                 int K, LinearOut out) {
    constexpr int XS = ST * ROWS * 16, RS = NT * NMB * 64;          // 16-byte words of a wave: x, partial sums
    __shared__ u32x4 lds[NW * (XS > RS ? XS : RS)];
    f32x4* red = (f32x4*)lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, kg = lane >> 4;
    const int m0 = blockIdx.y * 16 * NMB, KB = K / 128;
    // The workgroup's blocks of 16 outputs, each in its part; one past the last repeats it.
    const uint8_t* codes[NT];
    const uint16_t* scales[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        int nb = min((int)blockIdx.x * NT + i, (N + 15) / 16 - 1), t = 0;
        while (t < 2 && nb >= (W.rows[t] + 15) / 16) nb -= (W.rows[t++] + 15) / 16;
        const uint8_t* p = (const uint8_t*)W.p[t];
        codes[i] = p + (size_t)nb * KB * 1024;
        scales[i] = (const uint16_t*)(p + (size_t)((W.rows[t] + 15) / 16) * 8 * K) + (size_t)nb * (KB * GS) * 16;
    }
    f32x4 acc[NT][NMB];
#pragma unroll
    for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i][mb] = f32x4{};
    // x of 128 inputs in LDS: rows of 16 chunks of 16 bytes, chunk c of row r at place c ^ (r & 15).  A load is 4
    // rows; rows past M repeat the last one.
    u32x4* xl = lds + wave * XS;
    const uint16_t* xb = X + (size_t)m0 * K;
    const int rows = min(ROWS, M - m0);
    const int xr = ROWS == 4 ? col & 3 : col;          // the lane's row of a block
    uint32_t xa[4];                                    // addresses of its four chunks
#pragma unroll
    for (int w = 0; w < 4; ++w) xa[w] = (uint32_t)(uintptr_t)(xl + xr * 16 + ((4 * w + kg) ^ xr));
    uint32_t mask = 0x00780078u, one = 0x3F803F80u;
    asm("" : "+s"(mask), "+v"(one));
    const bf16x8 off = as_bf16x8(u32x4{0xBFC0BFC0u, 0xBFC0BFC0u, 0xBFC0BFC0u, 0xBFC0BFC0u});   // -1.5
    struct Codes {
        u32x4 c[NT];
        u32x2 s[NT][GS];
    };
    auto request = [&](Codes& S, int kb, int stg) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < ROWS / 4; ++j) {
            if (j && 4 * j >= rows) break;
            const int r = 4 * j + (lane >> 4);
            __builtin_amdgcn_global_load_lds(
                (gvoid_t*)(xb + (size_t)kb * 128 + (uint32_t)(min(r, rows - 1) * K + 8 * ((lane & 15) ^ (r & 15)))),
                (lvoid_t*)(xl + (stg * ROWS + 4 * j) * 16), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            S.c[i] = *(const u32x4*)(codes[i] + (size_t)kb * 1024 + (uint32_t)(16 * lane));
#pragma unroll
            for (int g = 0; g < GS; ++g)
                S.s[i][g] = *(const u32x2*)(scales[i] + (size_t)(kb * GS + g) * 16 + (uint32_t)(4 * kg));
        }
    };
    Codes now, next;
    if (ST == 2 && wave < KB) request(next, wave, 0);
    for (int kb = wave, stg = 0; kb < KB; kb += NW, stg ^= ST - 1) {
        if (ST == 1) request(next, kb, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // x is in LDS
        now = next;
        if (ST == 2 && kb + NW < KB) request(next, kb + NW, stg ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t at[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) at[w] = xa[w] + stg * (ROWS * 256);
        u32x4 x[NMB][4];
        lds_four<0>(at, x[0]);
        if constexpr (NMB > 1) lds_four<16 * 256>(at, x[1]);
        if constexpr (NMB > 2) lds_four<32 * 256>(at, x[2]);
        if constexpr (NMB > 3) lds_four<48 * 256>(at, x[3]);
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            f32x4 none[NMB];          // -1.5 sum_k x, for all outputs
#pragma unroll
            for (int w = g * (4 / GS); w < (g + 1) * (4 / GS); ++w)
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
                    none[mb] = mfma16x16x32(off, as_bf16x8(x[mb][w]), w % (4 / GS) ? none[mb] : f32x4{});
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                f32x4 part[NMB];
#pragma unroll
                for (int w = g * (4 / GS); w < (g + 1) * (4 / GS); ++w) {
                    const bf16x8 wf = widen4(now.c[i][w], mask, one);
#pragma unroll
                    for (int mb = 0; mb < NMB; ++mb)
                        part[mb] = mfma16x16x32(wf, as_bf16x8(x[mb][w]), w % (4 / GS) ? part[mb] : none[mb]);
                }
                const u32x2 s = now.s[i][g];
                const f32x4 sf = {bf(s[0]), __uint_as_float(s[0] & 0xFFFF0000u), bf(s[1]), __uint_as_float(s[1] & 0xFFFF0000u)};
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb) acc[i][mb] += sf * part[mb];
            }
        }
    }
    __syncthreads();       // x has been read
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) red[wave * RS + (i * NMB + mb) * 64 + lane] = acc[i][mb];
    __syncthreads();
    // Lane (col, kg) of block (i, mb): row 16 mb + col, outputs 4 kg .. + 3.
    for (int j = threadIdx.x; j < 64 * NT * NMB; j += 64 * NW) {
        const int ib = j >> 6, ln = j & 63, m = m0 + 16 * (ib % NMB) + (ln & 15);
        const int n = (blockIdx.x * NT + ib / NMB) * 16 + 4 * (ln >> 4);
        if (m >= M || n >= N) continue;
        f32x4 v = red[j];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += red[w * RS + j];
        v *= 16.f;
        const size_t at = (size_t)m * N + n;
        if (N % 4 == 0) {
            if (out.res) {
                if (out.res_f32) {
                    v += *(const f32x4*)((const float*)out.res + at);
                } else {
                    const u32x2 r = *(const u32x2*)((const uint16_t*)out.res + at);
                    v += f32x4{bf(r[0] & 0xFFFFu), bf(r[0] >> 16), bf(r[1] & 0xFFFFu), bf(r[1] >> 16)};
                }
            }
            if (out.y) *(u32x2*)(out.y + at) = u32x2{pack2bf(v[0], v[1]), pack2bf(v[2], v[3])};
            if (out.yf) *(f32x4*)(out.yf + at) = v;
            continue;
        }
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
    const int kb = blockIdx.y, nb = blockIdx.x, n = 16 * nb + i;
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
    uint16_t* scales = (uint16_t*)(out + (size_t)gridDim.x * 8 * K) + (nb * KB + kb) * GS * 16;
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

template <int NMB, int ROWS, int NT, int ST, int GS>
hipError_t launch(const uint16_t* x, const W4Rows& w, int M, int N, int K, const LinearOut& o, hipStream_t st) {
    const dim3 grid(((N + 15) / 16 + NT - 1) / NT, (M + 16 * NMB - 1) / (16 * NMB)), block(64 * NW);
    hipLaunchKernelGGL((linear_kernel<NMB, ROWS, NT, ST, GS>), grid, block, 0, st, x, w, M, N, K, o);
    return hipGetLastError();
}
// Blocks of 16 outputs a workgroup: as few as one workgroup on each of the 256 CUs allows, up to 4.  Every
// workgroup reads all of x, and a second one on some of the CUs costs as much as on all.  8192 inputs, us: 64 rows,
// 2048 outputs 13.9 with 1 block (16.2 with 2), 10240 21.8 with 3 (31.2 with 2), 14000 27.0 with 4 (33.0 with 2); 16
// rows, 4096 outputs 7.0 with 1 (8.3 with 2), 10240 11.1 with 3 (13.9 with 2).  11008 inputs, 1 row: 8192 outputs
// 9.8 with 2 (10.3 with 1), 14000 15.4 with 4 (16.5 with 1).
template <int NMB, int ROWS, int ST, int GS>
hipError_t launch_some(const uint16_t* x, const W4Rows& w, int M, int N, int K, const LinearOut& o, hipStream_t st) {
    const int64_t blocks = (int64_t)((N + 15) / 16) * ((M + 16 * NMB - 1) / (16 * NMB)), nt = (blocks + 255) / 256;
    if (nt <= 1) return launch<NMB, ROWS, 1, ST, GS>(x, w, M, N, K, o, st);
    if (nt == 2) return launch<NMB, ROWS, 2, ST, GS>(x, w, M, N, K, o, st);
    if (nt == 3) return launch<NMB, ROWS, 3, ST, GS>(x, w, M, N, K, o, st);
    return launch<NMB, ROWS, 4, ST, GS>(x, w, M, N, K, o, st);
}
template <int GS>
hipError_t launch(const uint16_t* x, const W4Rows& w, int M, int N, int K, const LinearOut& o, hipStream_t st) {
    if (M <= 4) return launch_some<1, 4, 2, GS>(x, w, M, N, K, o, st);
    if (M <= 16) return launch_some<1, 16, 2, GS>(x, w, M, N, K, o, st);
    if (M <= 32) return launch_some<2, 32, 2, GS>(x, w, M, N, K, o, st);
    return launch_some<4, 64, 1, GS>(x, w, M, N, K, o, st);
}

}  // namespace

size_t w4_bytes(int N, int K, int group) {
    const size_t nb = (N + 15) / 16;
    return nb * 8 * K + nb * 32 * (K / group);
}

bool w4_shape_ok(int K, int group) {
    return K >= 128 && K <= kMaxW4Rows && K % 128 == 0 && (group == 32 || group == 64 || group == 128);
}

hipError_t pack_w4(const uint16_t* w, int N, int K, int group, uint8_t* packed, hipStream_t st) {
    if (N < 1 || !w4_shape_ok(K, group)) return hipErrorInvalidValue;
    const dim3 grid((N + 15) / 16, K / 128), block(64);
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
    int N = 0;
    for (int t = 0; t < 3; ++t) {
        // Outputs are counted in blocks of 16 across the parts: only the last may end inside one.
        if (w.rows[t] < 0 || (t < 2 && w.rows[t + 1] && w.rows[t] % 16)) return hipErrorInvalidValue;
        N += w.rows[t];
    }
    if (!N) return hipErrorInvalidValue;
    if (group == 32) return launch<4>(x, w, M, N, K, o, st);
    if (group == 64) return launch<2>(x, w, M, N, K, o, st);
    return launch<1>(x, w, M, N, K, o, st);
}

}  // namespace kvp
