"""64-bit references of the operators on bf16 pages (append, attention with windows, page copies), on the host, from the
definitions in include/kvpipe.h; and what their roundings allow."""
from __future__ import annotations

import numpy as np
import torch

from lowbit_ref import D, PAGE, bf16, pages_for, rotate, rows_of, scattered  # noqa: F401
from paper_2608_15943_amd import binding as kb


def bits(x):
    """bf16 numbers (held in float32) as their 16 bits."""
    return (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def from_bits(u):
    return (np.ascontiguousarray(u).astype(np.uint32) << 16).view(np.float32)


class Cache:
    """Host copy of one producer's pools: K [g][n_pages][64][128], V [g][n_pages][128][64], as the 16 bits of bf16.  What was
    never written holds anything: NaN and infinities among it."""

    def __init__(self, g, n_pages, seed=0):
        rng = np.random.default_rng(seed)
        junk = np.array([0x7FC0, 0xFF80, 0x7F80, 0xFFFF, 0x7F7F], np.uint16)
        self.k, self.v = (junk[rng.integers(0, 5, s)] for s in ((g, n_pages, PAGE, D), (g, n_pages, D, PAGE)))
        self.g, self.n_pages = g, n_pages

    def put(self, table, b, n, kv):
        """Positions n, n + 1, ... of table row b: kv [2][T][g][128]."""
        for t in range(kv.shape[1]):
            page, r = table[b][(n + t) // PAGE], (n + t) % PAGE
            self.k[:, page, r], self.v[:, page, :, r] = bits(kv[0, t]), bits(kv[1, t])

    def values(self, table, b, n):
        """[2][n][g][128] of positions 0 .. n - 1; NaN where the table has no page."""
        pos = np.arange(n)
        page = np.asarray(table[b])[pos // PAGE]
        k = from_bits(self.k[:, page, pos % PAGE]).astype(np.float64)
        v = from_bits(self.v[:, page, :, pos % PAGE]).astype(np.float64)      # [n][g][128]
        out = np.stack([k.transpose(1, 0, 2), v])
        out[:, page < 0] = np.nan
        return out

    def to_device(self):
        return tuple(torch.from_numpy(t.view(np.int16).copy()).cuda().view(torch.bfloat16) for t in (self.k, self.v))

    def from_device(self, dev):
        c = Cache.__new__(Cache)
        c.k, c.v = (t.view(torch.int16).cpu().numpy().view(np.uint16) for t in dev)
        c.g, c.n_pages = self.g, self.n_pages
        return c

    def same(self, other):
        return np.array_equal(self.k, other.k) and np.array_equal(self.v, other.v)


def near(got, want, pair):
    """Rotated values rounded to bf16: half a step, 2^-8 of the value, and of the two products that the device rounds in 32
    bits (and the angle's cosine and sine) 2^-22 of the pair's larger magnitude."""
    return np.abs(got - want) <= 2.0**-8 * np.abs(want) + 2.0**-22 * 2 * pair


def check_append(before, after, table, lens, new, kv):
    """after: the device's pools when rows kv[b] [2][T][g][128] (rotated K, V; 64 bits) were appended to `before` at
    lens[b]: K near, V exactly, everything else as it was, bit for bit."""
    k0, v0 = before.k.copy(), before.v.copy()
    for b, (n, T) in enumerate(zip(lens, new)):
        if n < 0:
            continue
        for t in range(T):
            page, r = table[b][(n + t) // PAGE], (n + t) % PAGE
            got = from_bits(after.k[:, page, r]).astype(np.float64)
            want = kv[b][0, t]
            fin = np.isfinite(want)
            assert (near(got, want, np.abs(want[fin]).max(initial=0)) | ~fin).all(), (b, t)
            assert not np.isfinite(got[~fin]).any()
            k0[:, page, r] = after.k[:, page, r]
            v0[:, page, :, r] = bits(kv[b][1, t])
    assert np.array_equal(after.k, k0)
    assert np.array_equal(after.v, v0)


def sees(p, j, window=0, sinks=0):
    """Whether the row at position p sees position j (arrays)."""
    return (j <= p) & ((j > p - window) | (j < sinks) if window else True)


def attention(q, kv, n, a, window=0, sinks=0):
    """q [T][a][128] at positions n, n + 1, ... over kv [2][n + T][g][128]: output [T][a][128] and a bound on the device's
    difference.  Its weights are w_i = p_i (1 + e_i), |e_i| <= 2^-8 (half a step of bf16), in the sum above and below the line:
    sum w v / sum w - out = sum p_i e_i (v_i - out) / (1 + sum p_i e_i), at most 2^-8 / (1 - 2^-8) of sum p_i |v_i - out|, which
    is at most the root of sum p_i (v_i - out)^2 = sum p_i v_i^2 - out^2; the output's rounding is 2^-8 of it; and 1e-4 of
    sum p_i |v_i| for the 32-bit sums (of 128 products of a score, 128 * 2^-24 of their magnitudes, which the exponential turns
    into a share of a weight).  Positions that no row sees are taken out before anything is computed."""
    T, g = q.shape[0], kv.shape[2]
    out, tol = np.zeros((T, a, D)), np.zeros((T, a, D))
    p = n + np.arange(T)[:, None]
    see = sees(p, np.arange(n + T)[None], window, sinks)
    some = see.any(0)
    see, kv = see[:, some], kv[:, some]
    for h in range(a):
        k, v = kv[0][:, h * g // a], kv[1][:, h * g // a]
        s = np.where(see, q[:, h] @ k.T / np.sqrt(D), -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        o = w @ v
        spread = np.sqrt(np.maximum(w @ v**2 - o**2, 0))
        out[:, h] = o
        tol[:, h] = spread / 255 + 1e-4 * (w @ np.abs(v)) + 2.0**-8 * np.abs(o)
    return out, tol


def model(a, g, dev, n_pages, max_batch, max_seq, tau=(0,), base=10000.0):
    """A model on the device's bf16 pools: dev (K, V) of layer 0, or {producer: (K, V)}."""
    m = kb.Model(len(tau), a * D, a, g, D, kb.KVP_DTYPE_BF16, list(tau), max_batch=max_batch, max_seq=max_seq,
                 kv_capacity=(max_seq + 63) // 64 * 64, rope_base=base)
    for l, p in enumerate(tau):
        if l == p:
            k, v = dev if isinstance(dev, tuple) else dev[l]
            m.kvp_set_kv_pool(l, k.data_ptr(), v.data_ptr(), n_pages)
    return m
