"""The attention on bf16 pages at the ends of the range that include/kvpipe.h states: large queries, keys and values."""
import numpy as np
import pytest
import torch

import rows_ref as rr
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_gpu_rows import Case, D, _attention

pytestmark = pytest.mark.gpu

# One by one, listed, in equal parts; many columns whole and in parts.
CALLS = [([150, 0], [3, 5]), ([2100], [4]), ([3000, 70], [1, 1]), ([60, 1], [30, 20]), ([2500], [20])]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


def _case(lens, new, a, g, q, kv):
    c = Case(a, g, lens, new, seed=95)
    c.x[:, :a] = q
    for b, x in enumerate(kv):
        c.cache.put(c.table, b, 0, x)
    return c


@pytest.mark.parametrize("lens,new", CALLS)
@pytest.mark.parametrize("qexp,kexp", [(112, -91), (10, 11), (-80, 101)])
@pytest.mark.parametrize("window", [0, 1000])
def test_largest_queries_keys_and_values(lens, new, qexp, kexp, window):
    """Scores so large that one key takes everything: the output is that key's value, bit for bit."""
    say(f"[range] lens={lens} new={new} 2^{qexp} 2^{kexp} window={window}")
    rng = np.random.default_rng(5)
    rows = sum(new)
    q = rr.bf16((rng.uniform(0.5, 0.99, (rows, 4, D)) * rng.choice([-1, 1], (rows, 4, D))).astype(np.float32)) * np.float32(2.0**qexp)
    kv = []
    for n, T in zip(lens, new):
        x = rng.uniform(-1, 1, (2, n + T, 1, D))
        x[:, ::7, :, ::5] = 1.0
        kv.append(rr.bf16(x) * np.array([2.0**kexp, 2.0**80], np.float32)[:, None, None, None])
    c = _case(lens, new, 4, 1, q, kv)
    got = _attention(c, window=window, sinks=3 if window else 0)
    checked = 0
    for b, (n, T) in enumerate(zip(lens, new)):
        x = c.cache.values(c.table, b, n + T)[:, :, 0]
        for t in range(T):
            i = int(c.cu[b]) + t
            seen = np.flatnonzero(rr.sees(n + t, np.arange(n + t + 1), window, 3))
            s = q[i].astype(np.float64) @ x[0, seen].T / np.sqrt(D)
            top = np.argsort(-s, 1)[:, :2]
            mag = (np.abs(q[i].astype(np.float64)) @ np.abs(x[0, seen]).T).max() / np.sqrt(D)
            for h in range(4):
                # The 32-bit sums of two scores are off by 2 (D + 8) 2^-24 of their magnitudes at most; a weight of e^-60 is
                # below half a step of every value it is added to.
                if len(seen) > 1 and s[h, top[h, 0]] - s[h, top[h, 1]] < 2 * (D + 8) * 2.0**-24 * mag + 60:
                    continue
                checked += 1
                assert np.array_equal(got[i, h].astype(np.float64), x[1, seen[top[h, 0]]]), (i, h)
    assert np.isfinite(got).all() and checked >= 2 * rows


@pytest.mark.parametrize("lens,new", CALLS)
def test_large_values_under_ordinary_weights(lens, new):
    rng = np.random.default_rng(6)
    q = rr.bf16(rng.standard_normal((sum(new), 8, D)))
    kv = [rr.bf16(rng.uniform(-1, 1, (2, n + T, 2, D))) * np.array([1.0, 2.0**80], np.float32)[:, None, None, None]
          for n, T in zip(lens, new)]
    c = _case(lens, new, 8, 2, q, kv)
    got = _attention(c)
    for b, (n, T) in enumerate(zip(lens, new)):
        rows = slice(int(c.cu[b]), int(c.cu[b + 1]))
        want, tol = rr.attention(q[rows].astype(np.float64), c.cache.values(c.table, b, n + T), n, 8)
        assert (np.abs(got[rows] - want) <= tol).all(), b
