// The rotation of a row to its position (RoPE), and where an append's rows come from (device helpers shared by the
// 8-bit and the bf16 cache's appends).
#pragma once

#include "fp8_cache.h"

namespace kvp {
namespace {

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
    // Eight values as they are in memory; those in fp32, and as bf16.
    typedef u32x4 Raw;
    __device__ __forceinline__ Raw raw8(int row, int z, int col) const {
        return *(const u32x4*)(z == 0 ? q + (size_t)row * ldq + col : (z == 1 ? k : v) + (size_t)row * ldkv + col);
    }
    static __device__ __forceinline__ void widen(const Raw& w, float* x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ u32x4 bits(const Raw& w) { return w; }
    __device__ __forceinline__ uint16_t v1(int row, int col) const { return v[(size_t)row * ldkv + col]; }
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
    struct Raw {
        float x[8];
    };
    __device__ __forceinline__ Raw raw8(int row, int z, int col) const {
        Raw w;
        load<8>(row, z, col, w.x);
        return w;
    }
    static __device__ __forceinline__ void widen(const Raw& w, float* x) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = w.x[e];
    }
    static __device__ __forceinline__ u32x4 bits(const Raw& w) {
        return u32x4{pack2bf(w.x[0], w.x[1]), pack2bf(w.x[2], w.x[3]), pack2bf(w.x[4], w.x[5]), pack2bf(w.x[6], w.x[7])};
    }
    __device__ __forceinline__ uint16_t v1(int row, int col) const {
        float x;
        load<1>(row, 2, col, &x);
        return f2bf(x);
    }
};

}  // namespace
}  // namespace kvp
