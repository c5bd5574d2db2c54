"""64-bit references of the 8-bit paged cache and of the 4-bit weights, on the host, from the
definitions in include/kvpipe.h; and what their roundings allow."""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from paper_2608_15943_amd import binding as kb

D, PAGE, BLK = 128, 64, 16

# Values of the 256 e4m3 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF NaN.
_c = np.arange(256)
_e, _m = (_c >> 3) & 15, _c & 7
E4M3 = np.where(_e == 0, _m * 2.0**-9, (1 + _m / 8) * 2.0 ** (_e - 7.0)) * np.where(_c >= 128, -1.0, 1.0)
E4M3[(_c & 127) == 127] = np.nan
_POS = E4M3[:127]                         # 0 .. 448, ascending


def e4m3(x):
    """Nearest e4m3 numbers, ties to the even code; |x| <= 448."""
    ax = np.abs(x)
    hi = np.clip(np.searchsorted(_POS, ax), 1, 126)
    lo = hi - 1
    mid = (_POS[lo] + _POS[hi]) / 2
    up = (ax > mid) | ((ax == mid) & (hi % 2 == 0))
    return np.copysign(np.where(up, _POS[hi], _POS[lo]), x)


def scale_of(m):
    """Least power of two s >= 2^-100 with m <= 448 s."""
    if not np.isfinite(m):
        return np.nan
    e = -100
    if m > 0:
        e = max(-100, int(np.floor(np.log2(m))) - 10)
        while m > 448 * 2.0**e:
            e += 1
    return 2.0**e


def rotate(x, pos, base=10000.0):
    """x [..., 128] at one position."""
    ang = pos * base ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(ang), np.sin(ang)
    x1, x2 = x[..., : D // 2], x[..., D // 2:]
    return np.concatenate([x1 * c - x2 * s, x2 * c + x1 * s], -1)


class Cache:
    """Host copy of one producer's pools: codes as bytes, scales."""

    def __init__(self, g, n_pages, seed=0, garbage=True):
        rng = np.random.default_rng(seed)
        # What was never written holds anything: every byte, NaN codes and NaN scales among them.
        fill = (lambda *s: rng.integers(0, 256, s, dtype=np.uint8)) if garbage else (lambda *s: np.zeros(s, np.uint8))
        self.k, self.v = fill(g, n_pages, PAGE, D), fill(g, n_pages, PAGE // BLK, D, BLK)
        self.s = np.where(rng.random((g, n_pages, 2, 4)) < 0.5, np.nan, 1e30).astype(np.float32) if garbage else \
            np.ones((g, n_pages, 2, 4), np.float32)
        self.g, self.n_pages = g, n_pages

    def write(self, table, b, kv):
        """Fills positions 0 .. n - 1 of table row b with kv [2][n][g][128], a block at a time."""
        n = kv.shape[1]
        for j in range((n + BLK - 1) // BLK):
            page, blk = table[b][j * BLK // PAGE], j % (PAGE // BLK)
            rows = kv[:, j * BLK: (j + 1) * BLK]
            for z in range(2):
                for h in range(self.g):
                    x = rows[z][:, h]
                    s = scale_of(np.abs(x).max())
                    codes = code_of(e4m3(x / s))
                    if z == 0:
                        self.k[h, page, blk * BLK: blk * BLK + len(x)] = codes
                    else:
                        self.v[h, page, blk, :, : len(x)] = codes.T
                    self.s[h, page, z, blk] = s

    def values(self, table, b, n):
        """[2][n][g][128] of positions 0 .. n - 1."""
        out = np.zeros((2, n, self.g, D))
        for p in range(n):
            page, r, blk = table[b][p // PAGE], p % PAGE, p % PAGE // BLK
            out[0, p] = E4M3[self.k[:, page, r]] * self.s[:, page, 0, blk].astype(np.float64)[:, None]
            out[1, p] = E4M3[self.v[:, page, blk, :, p % BLK]] * self.s[:, page, 1, blk].astype(np.float64)[:, None]
        return out

    def to_device(self):
        return tuple(torch.from_numpy(t.copy()).cuda() for t in (self.k, self.v, self.s))

    def from_device(self, dev):
        c = Cache.__new__(Cache)
        c.k, c.v, c.s = (t.cpu().numpy() for t in dev)
        c.g, c.n_pages = self.g, self.n_pages
        return c


def code_of(v):
    """Bytes of e4m3 numbers."""
    c = np.searchsorted(_POS, np.abs(v)).astype(np.uint8)
    assert np.array_equal(_POS[c], np.abs(v))
    return c | (np.signbit(v).astype(np.uint8) << 7)


def check_append(before, after, table, lens, new, kv, exact_rows=None):
    """after: the device's pools when rows kv[b] [2][T][g][128] (rotated, 64 bits) were appended to `before` at lens[b].
    New codes are within half a step of value / scale (and the 2^-22 of the two products that the device rounds in 32 bits),
    old ones exactly rescaled, everything else as it was."""
    k0, v0, s0 = before.k.copy(), before.v.copy(), before.s.copy()
    for b, (n, T) in enumerate(zip(lens, new)):
        if n < 0 or T == 0:
            continue
        for j in range(n // BLK, (n + T - 1) // BLK + 1):
            page, blk = table[b][j * BLK // PAGE], j % (PAGE // BLK)
            lo, hi = max(n - j * BLK, 0), min(n + T - j * BLK, BLK)
            rows = kv[b][:, j * BLK + lo - n: j * BLK + hi - n]
            for z in range(2):
                for h in range(before.g):
                    x = rows[z][:, h]
                    f = scale_of(np.abs(x).max() if np.isfinite(x).all() else np.inf)
                    old = float(before.s[h, page, z, blk])
                    want = (np.nan if np.isnan(f) or np.isnan(old) else max(f, old)) if lo else f
                    got = float(after.s[h, page, z, blk])
                    assert got == want or (np.isnan(got) and np.isnan(want)), (b, j, z, h, got, want)
                    s0[h, page, z, blk] = got
                    o = (before.k[h, page, blk * BLK: (blk + 1) * BLK] if z == 0 else before.v[h, page, blk].T)
                    a = (after.k[h, page, blk * BLK: (blk + 1) * BLK] if z == 0 else after.v[h, page, blk].T)
                    e = o.copy()
                    if np.isnan(want):
                        e[:hi] = 0
                    else:
                        if lo and want > old:
                            e[:lo] = code_of(e4m3(E4M3[o[:lo]] * (old / want)))
                        u = x / want
                        half = np.maximum(2.0**-4 * np.abs(u), 2.0**-10)
                        slack = 2.0**-22 * np.sqrt(2) * np.abs(x).max() / want
                        assert (np.abs(E4M3[a[lo:hi]] - u) <= half + slack).all(), (b, j, z, h)
                        e[lo:hi] = a[lo:hi]
                    assert np.array_equal(a, e), (b, j, z, h)
                    if z == 0:
                        k0[h, page, blk * BLK: (blk + 1) * BLK] = e
                    else:
                        v0[h, page, blk] = e.T
    assert np.array_equal(after.k, k0) and np.array_equal(after.v, v0)
    assert np.array_equal(after.s, s0, equal_nan=True)


def attention(q, kv, n, a):
    """q [T][a][128] at positions n, n + 1, ... over kv [2][n + T][g][128]: output [T][a][128] and a bound on the device's
    difference.  Its weights are w_i = p_i (1 + e_i), |e_i| <= 2^-8 (half a step of bf16), in the sum above and below the line:
    sum w v / sum w - out = sum p_i e_i (v_i - out) / (1 + sum p_i e_i), at most 2^-8 / (1 - 2^-8) of sum p_i |v_i - out|; the
    output's rounding is 2^-8 of it; and 1e-4 for the 32-bit sums (of 128 products of a score, 128 * 2^-24 of their magnitudes,
    which the exponential turns into a share of a weight)."""
    T, g = q.shape[0], kv.shape[2]
    out, tol = np.zeros((T, a, D)), np.zeros((T, a, D))
    for t in range(T):
        k, v = kv[:, : n + t + 1]
        for h in range(a):
            s = k[:, h * g // a] @ q[t, h] / np.sqrt(D)
            p = np.exp(s - s.max())
            p /= p.sum()
            vh = v[:, h * g // a]
            out[t, h] = p @ vh
            tol[t, h] = p @ np.abs(vh - out[t, h]) / 255 + 1e-4 * (p @ np.abs(vh)) + 2.0**-8 * np.abs(out[t, h])
    return out, tol


# ---- 4-bit weights ------------------------------------------------------------------------------

def bf16(x):
    """float32 numbers rounded to bf16."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def w4_codes(w, group):
    """Codes [N][K] and scales [N][K / group] of weights w (bf16 numbers), in the 32-bit steps of the definition."""
    N, K = w.shape
    x = w.astype(np.float32).reshape(N, K // group, group)
    s = bf16(np.abs(x).max(-1) / np.float32(7))
    s[s < 2.0**-100] = 0
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.clip(np.rint(x / s[..., None]), -8, 7) + 8
    return np.where(s[..., None] > 0, c, 8).astype(np.int64).reshape(N, K), s


def w4_pack(codes, s):
    """The packed buffer (bytes) of include/kvpipe.h's layout."""
    N, K = codes.shape
    nb = (N + 15) // 16
    c = np.full((nb * 16, K), 8, np.int64)
    c[:N] = codes
    sc = np.zeros((nb * 16, s.shape[1]), np.float32)
    sc[:N] = s
    words = np.zeros((nb, K // 128, 4, 16, 4), np.uint32)          # [block][128 inputs][j][i][w]
    for e in range(8):
        sh = 4 * (e // 2) + 16 * (e % 2)
        part = c.reshape(nb, 16, K // 128, 4, 4, 8)[..., e]          # [block][i][kb][w][j]
        words |= (part.transpose(0, 2, 4, 1, 3) << sh).astype(np.uint32)
    sb = (sc.view(np.uint32) >> 16).astype(np.uint16).reshape(nb, 16, -1).transpose(0, 2, 1)
    return np.concatenate([np.ascontiguousarray(words).view(np.uint8).reshape(-1),
                           np.ascontiguousarray(sb).view(np.uint8).reshape(-1)])


def w4_weights(codes, s, group):
    return (codes - 8.0) * np.repeat(s.astype(np.float64), group, axis=1)


def linear_bound(x, y, s, group):
    """Half a step of bf16 on y, and the 32-bit sums: products of x with numbers below 2 (and with 1.5) times 16 s, at most 32
    products of an instruction, 8 instructions of a group, K / 1024 groups of a wave and 8 waves deep."""
    K = x.shape[1]
    depth = 32 * 8 + K // 128 + 8
    mag = np.abs(x) @ np.repeat(s.astype(np.float64), group, axis=1).T * 32
    return 2.0**-8 * np.abs(y) + depth * 2.0**-24 * mag


# ---- calls --------------------------------------------------------------------------------------

def rows_of(lens, new, table, cu=True, rows=None, max_new=None, max_pos=None):
    """(kvp_rows, its device tensors) of a call."""
    cus = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = dict(len=torch.tensor(lens, dtype=torch.int32).cuda(), pages=torch.from_numpy(np.asarray(table, np.int32).copy()).cuda())
    if cu:
        t["cu"] = torch.from_numpy(cus).cuda()
    last = max([n + T - 1 for n, T in zip(lens, new) if n >= 0 and T > 0], default=0)
    r = kb.kvp_rows(t["cu"].data_ptr() if cu else 0, t["len"].data_ptr(), t["pages"].data_ptr(), t["pages"].shape[1],
                    len(lens), int(cus[-1]) if rows is None else rows, max(max(new), 1) if max_new is None else max_new,
                    last if max_pos is None else max_pos)
    return r, t


def scattered(need, stride, spare, seed):
    """Table [B][stride] of distinct pages, -1 where none is needed, and the pages of the pool."""
    n_pages = sum(need) + spare
    perm = np.random.default_rng(seed).permutation(n_pages)
    tab, k = np.full((len(need), stride), -1, np.int32), 0
    for b, n in enumerate(need):
        tab[b, :n] = perm[k: k + n]
        k += n
    return tab, n_pages


def pages_for(lens, new):
    return [(max(n, 0) + T + PAGE - 1) // PAGE for n, T in zip(lens, new)]


def model8(a, g, cache_dev, n_pages, max_batch, max_seq, tau=(0,), base=10000.0):
    m = kb.Model(len(tau), a * D, a, g, D, kb.KVP_DTYPE_BF16, list(tau), max_batch=max_batch, max_seq=max_seq,
                 kv_capacity=(max_seq + 63) // 64 * 64, rope_base=base)
    for l, p in enumerate(tau):
        if l == p:
            k, v, s = cache_dev if isinstance(cache_dev, tuple) else cache_dev[l]
            m.kvp_set_kv_pool_fp8(l, k.data_ptr(), v.data_ptr(), s.data_ptr(), n_pages)
    return m
