// The 8-bit paged K/V cache: layout, scales, and the rows of a call (device helpers shared by the
// append and the attention).
//
// Pages hold 64 positions.  K codes [g][n_pages][64][128]: a position's 128 dimensions side by
// side.  V codes [g][n_pages][4][128][16]: 16 positions of one dimension side by side, so that
// both products of the attention read 16-byte runs along the axis they sum over.  Scales
// [g][n_pages][2][4] fp32: K and V, one for each block of 16 positions.  A code is an e4m3 number
// (1-4-3 bits, largest 448, no infinities), a scale a power of two: e4m3 has the same relative
// precision under any scale, so a scale between two powers of two would gain nothing, and with
// powers of two a block whose scale grows is rescaled without a second rounding (but for codes
// that fall below the smallest normal number, 2^-6 of the block's unit, 2^-15 of its largest
// value).
#pragma once

#include "common.h"
#include "kernels.h"

namespace kvp {

constexpr int kBlk = 16;                 // positions a scale
constexpr int kPageBlks = kPage / kBlk;
constexpr int kHead = 128;               // head dimension
constexpr int kMinScaleExp = -100;       // least exponent of a scale: its reciprocal stays finite

// Bytes of V block k of a page (2 KB each), and of a page of one head.
constexpr int kBlkBytes = kBlk * kHead, kPageBytes8 = kPage * kHead;

// The least power of two s with m <= 448 s, for m given as the bits of a non-negative float;
// NaN where m is infinite or NaN.
__device__ __forceinline__ float e4m3_scale(uint32_t m) {
    if (m >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    // 448 = 1.75 * 2^8.
    const int e = (int)(m >> 23) - 127 - 8 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(e, kMinScaleExp) + 127) << 23);
}

// Four values to e4m3 codes, nearest, ties to even; |v| <= 448.
__device__ __forceinline__ uint32_t e4m3_pack(float v0, float v1, float v2, float v3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v2, v3, w, true);
}

// Four codes times f (a power of two <= 1), to codes again.
__device__ __forceinline__ uint32_t e4m3_rescale(uint32_t c, float f) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    return e4m3_pack(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// New rows of sequence b: rows row0 .. row0 + n - 1 of the call's tensors, at positions len,
// len + 1, ...; only the first `act` of them lie at a position of the call's reach (none where
// the sequence is inactive).  Whatever the device arrays hold, rows stay in [0, rows) and
// positions in [0, max_pos].
struct SeqRows {
    int row0, n, len, act;
};
__device__ __forceinline__ SeqRows seq_rows(const NewRows& r, int b) {
    SeqRows s;
    s.len = r.len[b];
    if (r.cu) {
        s.row0 = min(max(r.cu[b], 0), r.rows);
        s.n = min(min(max(r.cu[b + 1], s.row0), r.rows) - s.row0, r.max_new);
    } else {
        s.row0 = b;
        s.n = 1;
    }
    s.act = s.len < 0 || s.len > r.max_pos ? 0 : min(s.n, r.max_pos + 1 - s.len);
    return s;
}

// Finds item x of the list in which sequence b has count(seq_rows(b)) items, in order of b: its
// sequence, that sequence's rows and first item.  False past the end.  All lanes of a wave
// together; every lane gets the answer.
template <class Count>
__device__ __forceinline__ bool find_item(const NewRows& r, int x, Count count, int* b, SeqRows* rows, int* first) {
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < r.B; b0 += 64) {
        SeqRows s{0, 0, 0, 0};
        int c = 0;
        if (b0 + lane < r.B) {
            s = seq_rows(r, b0 + lane);
            c = count(s);
        }
        int pre = c;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int v = __shfl_up(pre, off);
            if (lane >= off) pre += v;
        }
        const int total = __builtin_amdgcn_readlane(pre, 63);
        if (x < base + total) {
            const int w = __popcll(__ballot(base + pre <= x));   // lanes before the one that holds x
            *b = b0 + w;
            rows->row0 = __builtin_amdgcn_readlane(s.row0, w);
            rows->n = __builtin_amdgcn_readlane(s.n, w);
            rows->len = __builtin_amdgcn_readlane(s.len, w);
            rows->act = __builtin_amdgcn_readlane(s.act, w);
            *first = base + __builtin_amdgcn_readlane(pre - c, w);
            return true;
        }
        base += total;
    }
    return false;
}

__device__ __forceinline__ int page_of(const NewRows& r, int b, int pos) {
    return min(max(r.pt[(size_t)b * r.stride + pos / kPage], 0), r.n_pages - 1);
}

}  // namespace kvp
