"""Calls on 8-bit pages beside each other: different launches at once on streams of one model."""
import numpy as np
import pytest
import torch

import lowbit_ref as lr
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_gpu_fp8_cache import Case, _dev

pytestmark = pytest.mark.gpu
D = lr.D


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


def test_every_launch_at_once_on_streams_of_one_model():
    """Four calls of one model over one pool, each on a stream and with a workspace of its own, whose sizes pick different
    launches: blocks of rows by list with a join (long contexts), blocks one by one (short prompts), single tokens by list with
    a join, single tokens in one launch.  Each equals its bits alone, every time."""
    calls = [([2500, 64], [3, 40]), ([0, 5, 0], [150, 200, 90]), ([6000, 9000], [1, 1]), ([300, 17, 200], [1, 1, 1])]
    lens, new = [n for c in calls for n in c[0]], [t for c in calls for t in c[1]]
    c = Case(8, 2, lens, new, seed=43)
    rng = np.random.default_rng(44)
    for b, (n, T) in enumerate(zip(lens, new)):
        c.cache.write(c.table, b, rng.standard_normal((2, n + T, 2, D)))
    dev = c.cache.to_device()
    m = lr.model8(8, 2, dev, c.cache.n_pages, 3, 500)
    work, b0, r0 = [], 0, 0
    for ls, ns in calls:
        B, rows = len(ls), sum(ns)
        r, keep = lr.rows_of(ls, ns, c.table[b0: b0 + B])
        q = _dev(c.x[r0: r0 + rows, :8].reshape(rows, -1))
        n = m.kvp_workspace_size(kb.KVP_PHASE_STEP_FP8, B, rows)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        work.append((r, keep, q, ws, n, range(b0, b0 + B), r0, torch.cuda.Stream()))
        b0, r0 = b0 + B, r0 + rows

    def attend(w, out, st):
        m.kvp_attention_fp8(0, w[2].data_ptr(), w[0], out.data_ptr(), w[3].data_ptr(), w[4], st.cuda_stream)

    alone = []
    for w in work:
        out = torch.full_like(w[2], float("nan"))
        attend(w, out, torch.cuda.current_stream())
        torch.cuda.synchronize()
        alone.append(out)
        got = out.float().cpu().numpy().reshape(-1, 8, D)
        for b in w[5]:
            rows = slice(int(c.cu[b]) - w[6], int(c.cu[b + 1]) - w[6])
            want, tol = lr.attention(c.x[c.cu[b]: c.cu[b + 1], :8].astype(np.float64), c.cache.values(c.table, b, lens[b] + new[b]),
                                     lens[b], 8)
            assert (np.abs(got[rows] - want) <= tol).all(), b
    outs = [[torch.full_like(w[2], float("nan")) for _ in range(6)] for w in work]
    torch.cuda.synchronize()
    for i in range(6):
        for w, o in zip(work, outs):
            attend(w, o[i], w[7])
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a, x) for x in o)
