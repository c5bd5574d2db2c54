"""The 8-bit attention at the ends of what include/kvpipe.h promises: queries in two 8-bit parts."""
import numpy as np
import pytest
import torch

import lowbit_ref as lr
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_query_split import bf16_up_to_448, split

pytestmark = pytest.mark.gpu
D = lr.D


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


def _attend(q, kv, lens, new, max_new=None):
    """kvp_attention_fp8 of q [rows][a][128] (bf16 numbers), the rows of sequence b behind lens[b] positions, over the cached
    kv[b] [2][lens[b] + new[b]][g][128]; the output and the cache's values."""
    a, g = q.shape[1], kv[0].shape[2]
    need = lr.pages_for(lens, new)
    table, n_pages = lr.scattered(need, max(need), 2, 1)
    cache = lr.Cache(g, n_pages, 2)
    for b, x in enumerate(kv):
        cache.write(table, b, x)
    dev = cache.to_device()
    m = lr.model8(a, g, dev, n_pages, len(lens), max(q.shape[0], max_new or 1))
    r, keep = lr.rows_of(lens, new, table, max_new=max_new)
    qd = torch.from_numpy(np.ascontiguousarray(q, dtype=np.float32)).to(torch.bfloat16).cuda()
    out = torch.full_like(qd, float("nan"))
    n = m.kvp_workspace_size(kb.KVP_PHASE_STEP_FP8, len(lens), q.shape[0])
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    m.kvp_attention_fp8(0, qd.data_ptr(), r, out.data_ptr(), ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), [cache.values(table, b, x.shape[1]) for b, x in enumerate(kv)]


def _small_value(exact):
    """A value in units of a scale whose largest is 225: the least kept well by two e4m3 parts of those that are exact, or the
    farthest from its two parts."""
    if exact:
        return 206 / 2048
    x = bf16_up_to_448()
    x = x[x < 2.0**-6]
    return float(x[(split(x) - x.double()).abs().argmax()])


@pytest.mark.parametrize("T", [12, 40])
@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("unit", [0, -60, 40])
def test_queries_of_two_parts(T, exact, unit):
    """Keys of two kinds with nearly the same score, one from the query's largest value and one from 127 small ones: a small
    value that is off shifts the weights between them.  Values of 1 and -1 make the output the difference of the weights."""
    a, n = 4, 100
    small = _small_value(exact)
    q = np.full((T, a, D), small)
    q[..., 0] = 225.0
    c = 176.0 if exact else 448.0
    k0 = lr.e4m3(np.array(127 * small * c / 225 * 2**4))[()] / 2**4       # a number of 4 bits
    kv = np.zeros((2, n + T, 1, D))
    kv[0, ::2, 0, 1:], kv[0, 1::2, 0, 0] = c, k0
    kv[1, ::2], kv[1, 1::2] = 1.0, -1.0
    got, held = _attend(q * 2.0**unit, [kv * np.array([2.0**-unit, 1.0])[:, None, None, None]], [n], [T])
    assert np.array_equal(held[0][0] * 2.0**unit, kv[0]) and np.array_equal(held[0][1], kv[1])
    want, tol = lr.attention(q, kv, n, a)
    # Two scores are each off by their 32-bit sums and, where values are not exact, by the header's 2^-21 of the largest value
    # times the keys; the share of a weight moves by that (at most, of the two kinds' difference 2 P (1 - P) <= 1/2 each).
    shift = 2 * 128 * 2.0**-24 * 225 * k0 / np.sqrt(D) + (0 if exact else 2.0**-21 * 225 * 127 * c / np.sqrt(D))
    e = np.abs(got - want).max()
    say(f"[two parts] T={T} exact={exact} unit={unit}: off {e:.2e}, allowed {tol.max() + shift:.2e}")
    assert (np.abs(got - want) <= tol + shift).all()
