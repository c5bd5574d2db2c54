"""Calls on 8-bit pages beside each other: different launches at once on streams of one model, graphs that share a workspace,
and what a prompt at once and in chunks leaves in the cache."""
import numpy as np
import pytest
import torch

import lowbit_ref as lr
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_gpu_fp8_cache import Case, Stack, _dev, _normal

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


def _held(s, l, n):
    """[2][n][g][128] values and [2][n][g] scales of sequence 0 in layer l's pools."""
    c = lr.Cache(s.g, 1).from_device(s.dev[l])
    pos = np.arange(n)
    page, blk = s.table[0][pos // lr.PAGE], pos % lr.PAGE // lr.BLK
    return c.values(s.table, 0, n), np.stack([c.s[:, page, z, blk].T for z in range(2)]).astype(np.float64)


@pytest.mark.parametrize("rows,chunks", [(64, (0, 16, 48, 64)), (61, (0, 13, 40, 61)), (70, (0, 16, 48, 70))])
def test_prompt_at_once_and_in_chunks_fill_the_cache_alike(rows, chunks):
    """Up to 64 rows the projections stay in 32 bits until a value is rounded to its code, so layer 0's caches differ where
    another order of sums (or, of chunks that begin inside a block, a scale that grew on the way) tips a rounding; past 64 rows
    the prompt's are rounded to bf16 in between.  Layer 1 gets what differs in layer 0's outputs, which stacks of that layer
    alone show."""
    rng = np.random.default_rng(45)
    x = _normal(rng, rows, 512)

    def runs(tau):
        one, two = Stack(4, 2, tau, 1, 4, seed=46), Stack(4, 2, tau, 1, 4, seed=46)
        y1 = one.step(x, [0], [rows])
        y2 = np.concatenate([two.step(x[lo:hi], [lo], [hi - lo]) for lo, hi in zip(chunks, chunks[1:])])
        return one, two, y1, y2

    one, two, _, _ = runs((0, 1))
    alone, _, y1, y2 = runs((0,))
    assert all(np.array_equal(alone.w[0][k], one.w[0][k]) for k in "qkvo") and np.array_equal(alone.table, one.table)
    for l, (inp, diff) in enumerate(((x, np.zeros_like(x)), (y1, np.abs(y1 - y2)))):
        (v1, s1), (v2, s2) = _held(one, l, rows), _held(two, l, rows)
        assert np.isfinite(v1).all() and np.isfinite(v2).all()
        assert (np.maximum(s1, s2) / np.minimum(s1, s2) <= 2).all()
        # The values before their codes, [2][rows][g][128]: the inputs' differences times the weights, another order of 512
        # products (2 x 512 x 2^-24 of their magnitudes), 2^-8 of them where they are rounded to bf16; a rotation adds a pair's.
        delta = np.zeros((2, rows, 2, D))
        for z, k in enumerate("kv"):
            w = one.w[l][k].T
            moved, mag = diff @ np.abs(w), np.abs(inp) @ np.abs(w)
            rounded = 2.0**-8 * (np.abs(inp @ w) + moved + 2.0**-14 * mag) if rows > 64 else 0
            delta[z] = (moved + 2.0**-14 * mag + rounded).reshape(rows, 2, D)
        delta[0] += np.roll(delta[0], D // 2, -1)
        # Codes: half a step each, 2^-4 of the value or 2^-10 of the scale; a scale that grows rounds the earlier ones again.
        top, s = np.maximum(np.abs(v1), np.abs(v2)), np.maximum(s1, s2)[..., None]
        tol = delta + 3 * np.maximum(2.0**-4 * 1.1 * top, 2.0**-10 * s)
        e = np.abs(v1 - v2)
        say(f"[chunks] rows={rows} layer {l}: {(e > 0).mean():.4f} of the values differ, {(e / tol).max():.3f} of what may be")
        assert (e <= tol).all(), l
        if l == 0 and rows == 64:      # chunks end at block ends: another order of sums alone
            assert (e > 0).mean() <= 0.01


def test_two_graphs_share_a_workspace():
    """Two captured steps on one workspace, one of single tokens and one of chunks, replayed in turn and between eager calls:
    each leaves the outputs and caches of the same eager call."""
    s = Stack(4, 2, (0, 0), 3, 8, seed=47)
    rng = np.random.default_rng(48)
    s.step(_normal(rng, 140, s.h), [0, 0, 0], [30, 100, 10])
    start = {l: [t.clone() for t in d] for l, d in s.dev.items()}
    calls = [([30, 100, 10], [1, 1, 1]), ([30, 100, 10], [40, 3, 29])]
    n = max(s.m.kvp_workspace_size(kb.KVP_PHASE_STEP_FP8, 3, sum(t)) for _, t in calls)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    state = []
    for lens, new in calls:
        r, keep = lr.rows_of(lens, new, s.table)
        x = _dev(_normal(rng, sum(new), s.h))
        state.append((r, keep, x, torch.empty_like(x)))

    def run(i):
        r, _, x, y = state[i]
        s.m.kvp_step_fp8(x.data_ptr(), r, y.data_ptr(), ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)

    def result(f, i):
        for l, d in s.dev.items():
            for t, u in zip(d, start[l]):
                t.copy_(u)
        state[i][3].fill_(float("nan"))
        f()
        torch.cuda.synchronize()
        return state[i][3].clone(), [t.clone() for d in s.dev.values() for t in d]

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        run(0), run(1)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            run(i)
    for rep in range(3):
        for i, g in enumerate(graphs):
            state[i][2].copy_(_dev(_normal(rng, sum(calls[i][1]), s.h)))
            want, got = result(lambda: run(i), i), result(g.replay, i)
            assert torch.isfinite(want[0]).all() and torch.equal(want[0], got[0]), (rep, i)
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want[1], got[1])), (rep, i)
