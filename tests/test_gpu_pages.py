"""Pages of the cache copied, shared, trimmed and compacted, and the step on bf16 pages that uses them, on the GPU: whole runs
as a serving program makes them, against the 64-bit references (rows_ref.py)."""
import numpy as np
import pytest
import torch

import lowbit_ref as lr
import rows_ref as rr
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_gpu_rows import Case, _attention, _check_attention, _dev, _fill, _normal

pytestmark = pytest.mark.gpu
D = rr.D


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


# ---- copies ----------------------------------------------------------------------------------------

def _pools(rng, g, n_pages, fp8):
    """Any bits."""
    def any_bits(*shape):
        return torch.from_numpy(rng.integers(0, 256, shape, dtype=np.uint8)).cuda()

    if fp8:
        return any_bits(g, n_pages, 64 * D), any_bits(g, n_pages, 64 * D), any_bits(g, n_pages, 32)
    return any_bits(g, n_pages, 128 * D), any_bits(g, n_pages, 128 * D)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("g,sizes,n", [(1, [2], 1), (8, [40, 40, 40], 17), (3, [10, 7, 10], 4), (2, [300], 150), (1, [5] * 70, 2)])
def test_copy_pages(fp8, g, sizes, n):
    """Every producer's pools, of different sizes too, more producers than a launch takes, consumers between them; pairs that
    are none, that lie outside a pool, a page with itself, one source of several targets."""
    say(f"[copy] fp8={fp8} g={g} pools={sizes[:4]} n={n}")
    rng = np.random.default_rng(n + g)
    tau = []
    for _ in sizes:
        tau += [len(tau)] * 2                       # a producer and a consumer
    m = kb.Model(len(tau), 2 * g * D, 2 * g, g, D, kb.KVP_DTYPE_BF16, tau, max_batch=1, max_seq=64, kv_capacity=64)
    pools = [_pools(rng, g, k, fp8) for k in sizes]
    for i, (p, k) in enumerate(zip(pools, sizes)):
        (m.kvp_set_kv_pool_fp8 if fp8 else m.kvp_set_kv_pool)(2 * i, *(t.data_ptr() for t in p), k)
    perm = rng.permutation(max(sizes))
    src, dst = perm[:n].astype(np.int64), perm[n: 2 * n].astype(np.int64)
    if n > 3:
        src[1] = src[0]
        dst[2] = src[2]                             # itself
        src[3] = -1
    src = np.concatenate([src, [0, 1 << 30, -5]])
    dst = np.concatenate([dst, [-1, 0, -7]])
    want = [[t.clone() for t in p] for p in pools]
    for p, k in zip(want, sizes):
        for s, d in zip(src, dst):
            if 0 <= s < k and 0 <= d < k:
                for t in p:
                    t[:, d] = t[:, s]
    s, d = _i32(src), _i32(dst)
    call = m.kvp_copy_pages_fp8 if fp8 else m.kvp_copy_pages
    call(s.data_ptr(), d.data_ptr(), len(src), _stream())
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        assert all(torch.equal(x, y) for x, y in zip(p, w))


def test_copy_pages_past_4_gib_and_of_unset_producers():
    """Pages whose bytes lie past 2^32; a producer without pools is left out."""
    m = kb.Model(2, 8 * D, 8, 8, D, kb.KVP_DTYPE_BF16, [0, 1], max_batch=1, max_seq=64, kv_capacity=64)
    n_pages = 40000
    k, v = (torch.zeros(8, n_pages, 64 * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m.kvp_set_kv_pool(1, k.data_ptr(), v.data_ptr(), n_pages)
    k[:, 39998] = torch.randn(8, 64 * D, device="cuda").bfloat16()
    v[:, 3] = torch.randn(8, 64 * D, device="cuda").bfloat16()
    s, d = _i32([39998, 3]), _i32([1, 39997])
    m.kvp_copy_pages(s.data_ptr(), d.data_ptr(), 2, _stream())
    torch.cuda.synchronize()
    assert torch.equal(k[:, 1], k[:, 39998]) and torch.equal(v[:, 39997], v[:, 3])
    assert k[:, 1].abs().sum() > 0 and int((k.view(8, n_pages, -1)[:, :, 0] != 0).sum()) <= 16


# ---- the stack -------------------------------------------------------------------------------------

class Stack:
    """A stack on bf16 pages on the device, and the same on the host in 64 bits with K and V rounded as the cache holds them."""

    def __init__(self, a, g, tau, n_pages, B, seed, w4=None, max_seq=256, windows=()):
        rng = np.random.default_rng(seed)
        self.a, self.g, self.tau, self.h, self.n_pages = a, g, tau, a * D, n_pages
        self.m = kb.Model(len(tau), self.h, a, g, D, kb.KVP_DTYPE_BF16, list(tau), max_batch=B, max_seq=max_seq, kv_capacity=
                          (max_seq + 63) // 64 * 64)
        self.windows = [windows[l] if l < len(windows) else (0, 0) for l in range(len(tau))]
        self.dev, self.w, self.keep = {}, [], []
        for l, p in enumerate(tau):
            w = {"q": _normal(rng, self.h, self.h, scale=0.04), "o": _normal(rng, self.h, self.h, scale=0.04)}
            if l == p:
                w["k"], w["v"] = (_normal(rng, g * D, self.h, scale=0.04) for _ in range(2))
                self.dev[l] = rr.Cache(g, n_pages, seed + l).to_device()
                self.m.kvp_set_kv_pool(l, *(t.data_ptr() for t in self.dev[l]), n_pages)
            t = {k: _dev(v) for k, v in w.items()}
            at = lambda k: t[k].data_ptr() if k in t else 0  # noqa: E731
            if w4 is None or l % 2:         # with w4, the even layers have 4-bit weights and nothing else
                self.m.kvp_set_layer(l, at("q"), at("k"), at("v"), at("o"))
            else:
                for k, x in list(w.items()):
                    codes, s = lr.w4_codes(x, w4)
                    w[k] = lr.w4_weights(codes, s, w4)
                    buf = torch.empty(kb.kvp_w4_bytes(*x.shape, w4), dtype=torch.uint8, device="cuda")
                    kb.kvp_pack_w4(t[k].data_ptr(), *x.shape, w4, buf.data_ptr(), _stream())
                    torch.cuda.synchronize()
                    t[k] = buf
                self.m.kvp_set_layer_w4(l, at("q"), at("k"), at("v"), at("o"), w4)
            if self.windows[l][0]:
                self.m.kvp_set_layer_window(l, *self.windows[l])
            self.w.append({k: v.astype(np.float64) for k, v in w.items()})
            self.keep.append(t)
        self.kv = {}                       # (producer, sequence) -> [2][n][g][128]

    def step(self, x, lens, new, table, cu=True, rows=None, ws=None):
        """x [rows][h] (bf16 numbers) -> y of the device."""
        r, keep = rr.rows_of(lens, new, table, cu=cu, rows=rows)
        n = self.m.kvp_workspace_size(kb.KVP_PHASE_STEP, len(lens), r.rows)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        dx = _dev(x)
        y = torch.full_like(dx, float("nan"))
        self.m.kvp_step(dx.data_ptr(), r, y.data_ptr(), ws.data_ptr(), n, _stream())
        torch.cuda.synchronize()
        return y.float().cpu().numpy().astype(np.float64)

    def host(self, x, lens, new, seqs=None):
        """The same step on the host; seqs: the sequences' names."""
        y = x.astype(np.float64).copy()
        cu = np.concatenate([[0], np.cumsum(new)])
        for l, p in enumerate(self.tau):
            w = self.w[l]
            for i, (n, T) in enumerate(zip(lens, new)):
                b = i if seqs is None else seqs[i]
                if n < 0 or not T:
                    continue
                rows = slice(cu[i], cu[i] + T)
                z = y[rows]
                q = (z @ w["q"].T).reshape(T, self.a, D)
                q = np.stack([rr.rotate(q[t], n + t) for t in range(T)])
                if l == p:
                    k = (z @ w["k"].T).reshape(T, self.g, D)
                    k = np.stack([rr.rotate(k[t], n + t) for t in range(T)])
                    v = (z @ w["v"].T).reshape(T, self.g, D)
                    old = self.kv.get((l, b), np.zeros((2, 0, self.g, D)))[:, :n]
                    self.kv[l, b] = np.concatenate([old, rr.bf16(np.stack([k, v])).astype(np.float64)], 1)
                out, _ = rr.attention(q, self.kv[p, b], n, self.a, *self.windows[l])
                y[rows] = z + out.reshape(T, -1) @ w["o"].T
        return y


def _close(got, want, what):
    e = np.abs(got - want).max() / np.abs(want).max()
    say(f"  {what}: {e:.3e}")
    assert e <= 2e-2, what


def _scattered(B, stride, seed):
    perm = np.random.default_rng(seed).permutation(B * stride + 3)
    return perm[: B * stride].reshape(B, stride).astype(np.int32), B * stride + 3


@pytest.mark.parametrize("a,g,tau,w4,windows", [
    (4, 2, (0, 0, 2), None, ()), (4, 1, (0, 0, 0, 3), None, ()), (4, 2, (0, 0, 2, 2), 64, ()),
    (4, 2, (0, 0, 2, 2), None, ((0, 0), (30, 2), (7, 0)))])
def test_step_chunks_and_tokens(a, g, tau, w4, windows):
    """Prompts in chunks beside single tokens, then single tokens: every call against the host's stack; layers with windows
    and without."""
    say(f"[step] a={a} g={g} tau={tau} w4={w4} windows={windows}")
    B = 3
    table, n_pages = _scattered(B, 5, 30)
    s = Stack(a, g, tau, n_pages, B, seed=30, w4=w4, windows=windows)
    rng = np.random.default_rng(31)
    lens = [0, 0, -1]
    for i, new in enumerate(([37, 5, 2], [20, 1, 0], [66, 30, 0], [1, 1, 1], [1, 1, 1], [5, 3, 2])):
        if i == 4:
            lens[2] = 0
        x = _normal(rng, sum(new), s.h)
        got, want = s.step(x, lens, new, table), s.host(x, lens, new)
        _close(got, want, f"lens={lens} new={new}")
        cu = np.cumsum([0] + new)
        if lens[2] < 0:      # inactive: passes through
            assert np.array_equal(got[cu[2]: cu[3]], x[cu[2]: cu[3]].astype(np.float64))
        lens = [n + t if n >= 0 else n for n, t in zip(lens, new)]


def test_step_beside_the_other_calls_on_the_same_pages():
    """kvp_prefill_paged, kvp_decode_step_paged and kvp_step go on from each other's cache, and give what the others would."""
    B, S = 2, 70
    table, n_pages = _scattered(B, 3, 40)
    s = Stack(4, 2, (0, 0, 2), n_pages, B, seed=40)
    rng = np.random.default_rng(41)
    x = _normal(rng, B * S, s.h)
    want = s.host(x, [0] * B, [S] * B)
    dx, pt = _dev(x), _i32(table)
    y = torch.empty_like(dx)
    n = max(s.m.kvp_workspace_size(ph, B, S) for ph in (kb.KVP_PHASE_PREFILL, kb.KVP_PHASE_DECODE))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    s.m.kvp_prefill_paged(dx.data_ptr(), y.data_ptr(), B, S, pt.data_ptr(), 3, ws.data_ptr(), n, _stream())
    torch.cuda.synchronize()
    _close(y.float().cpu().numpy(), want, "prefill")
    _close(s.step(x, [0] * B, [S] * B, table), want, "step as a prefill")
    for i in range(3):
        x1 = _normal(rng, B, s.h)
        want = s.host(x1, [S + i] * B, [1] * B)
        d1, lens = _dev(x1), _i32([S + i] * B)
        y1 = torch.empty_like(d1)
        s.m.kvp_decode_step_paged(d1.data_ptr(), lens.data_ptr(), S + i, pt.data_ptr(), 3, y1.data_ptr(), B, ws.data_ptr(), n,
                                  _stream())
        torch.cuda.synchronize()
        _close(y1.float().cpu().numpy(), want, "decode step")
        _close(s.step(x1, [S + i] * B, [1] * B, table, cu=False), want, "step of one row each")


def test_step_rows_of_no_sequence_pass_through():
    table, n_pages = _scattered(2, 4, 32)
    s = Stack(4, 2, (0, 0), n_pages, 2, seed=32)
    x = _normal(np.random.default_rng(33), 80, s.h)
    got = s.step(x, [0, 0], [30, 45], table, rows=80)
    assert np.array_equal(got[75:], x[75:].astype(np.float64))
    want = s.host(x[:75], [0, 0], [30, 45])
    _close(got[:75], want, "rows")


@pytest.mark.parametrize("fp8", [False, True])
def test_fork_own_copy_and_append(fp8):
    """One prompt, three continuations of it: pages shared, the last one copied when its holder writes, as a program runs it
    through the pager, kvp_copy_pages and the step; each continuation reads as if it had a cache of its own."""
    say(f"[fork] fp8={fp8}")
    seqs, stride, pool = 4, 5, 14
    p = kb.Pager(pool, seqs, stride)
    rng = np.random.default_rng(50)
    s = Stack(4, 2, (0, 0, 2), pool, seqs, seed=50)
    if fp8:
        s.dev8 = {l: lr.Cache(2, pool, l).to_device() for l in s.dev}
        for l, t in s.dev8.items():
            s.m.kvp_set_kv_pool_fp8(l, *(x.data_ptr() for x in t), pool)

    def step(x, lens, new, ids):
        r, keep = rr.rows_of(lens, new, p.rows(ids))
        phase = kb.KVP_PHASE_STEP_FP8 if fp8 else kb.KVP_PHASE_STEP
        n = s.m.kvp_workspace_size(phase, len(ids), r.rows)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        dx = _dev(x)
        y = torch.empty_like(dx)
        (s.m.kvp_step_fp8 if fp8 else s.m.kvp_step)(dx.data_ptr(), r, y.data_ptr(), ws.data_ptr(), n, _stream())
        torch.cuda.synchronize()
        return y.float().cpu().numpy()

    def own(seq, lo, hi):
        src, dst = p.own(seq, lo, hi)
        if src.size:
            a, b = _i32(src), _i32(dst)
            (s.m.kvp_copy_pages_fp8 if fp8 else s.m.kvp_copy_pages)(a.data_ptr(), b.data_ptr(), src.size, _stream())
            torch.cuda.synchronize()
        return src.size

    x = _normal(rng, 150, s.h)
    p.reserve(0, 150)
    want = s.host(x, [0], [150], seqs=[0])
    tol = 6e-2 if fp8 else 2e-2      # the host's cache is not held in 8 bits: e4m3 keeps 4 bits, an error of 2^-4 a value
    e = np.abs(step(x, [0], [150], [0]) - want).max() / np.abs(want).max()
    assert e <= tol, e
    for t in (1, 2, 3):
        p.fork(0, t, 150)
        for l in s.dev:
            s.kv[l, t] = s.kv[l, 0].copy()
    assert p.free_pages() == pool - 3
    lens, copies = [150] * 4, 0
    for i in range(8):
        new = [1, 3, 2, 4]
        for t in range(4):
            p.reserve(t, lens[t] + new[t])
            copies += own(t, lens[t], lens[t] + new[t])
        x = _normal(rng, sum(new), s.h)
        got, want = step(x, lens, new, [0, 1, 2, 3]), s.host(x, lens, new, seqs=[0, 1, 2, 3])
        e = np.abs(got - want).max() / np.abs(want).max()
        say(f"  continuation {i}: {e:.3e}")
        assert e <= tol, e
        lens = [n + t for n, t in zip(lens, new)]
    assert copies == 3 and p.free_pages() == pool - 3 - 3      # the last of the four holders keeps the page itself
    tab = p.rows([0, 1, 2, 3])
    assert (tab[:, :2] == tab[0, :2]).all() and len(set(tab[:, 2].tolist())) == 4


def test_windowed_generation_on_few_pages():
    """A long generation through layers with windows on a pool that could not hold it: pages are trimmed behind the widest
    window, handed out again, and at times compacted; every step as the host's."""
    say("[windowed generation]")
    window, sinks, pool, stride = 130, 3, 8, 12
    s = Stack(4, 2, (0, 0, 2), pool, 2, seed=60, windows=((window, sinks), (60, 0), (window, sinks)))
    p = kb.Pager(pool, 2, stride)
    rng = np.random.default_rng(61)
    lens = [0, 0]
    moved = 0
    for i, new in enumerate([[70, 20]] + [[37, 11]] * 15):
        for b in range(2):
            p.trim(b, sinks, lens[b] - window + 1)
            p.reserve(b, lens[b] + new[b])
        if i % 4 == 3:
            src, dst = p.compact(pool)
            moved += src.size
            if src.size:
                a, b_ = _i32(src), _i32(dst)
                s.m.kvp_copy_pages(a.data_ptr(), b_.data_ptr(), src.size, _stream())
        x = _normal(rng, sum(new), s.h)
        _close(s.step(x, lens, new, p.rows([0, 1])), s.host(x, lens, new), f"lens={lens}")
        lens = [n + t for n, t in zip(lens, new)]
    assert lens[0] > 600 and lens[0] + lens[1] > 64 * pool
    say(f"  {moved} pages moved")


def test_every_launch_at_once_on_streams_of_one_model():
    """Calls of one model over one pool, each on a stream and with a workspace of its own, whose sizes pick different launches,
    with a window and without (layer 1 has one).  Each equals its bits alone, every time."""
    calls = [([2500, 64], [3, 40], 0), ([0, 5, 0], [150, 200, 90], 1), ([6000, 9000], [1, 1], 0), ([300, 17, 200], [1, 1, 1], 1),
             ([6000, 3000], [30, 70], 1), ([5000, 8000, 100], [1, 1, 1], 1)]
    lens, new = [n for c in calls for n in c[0]], [t for c in calls for t in c[1]]
    c = Case(8, 2, lens, new, seed=43)
    _fill(c)
    dev = c.cache.to_device()
    m = rr.model(8, 2, {0: dev}, c.cache.n_pages, 3, 500, tau=(0, 0))
    m.kvp_set_layer_window(1, 3000, 4)
    work, b0, r0 = [], 0, 0
    for ls, ns, layer in calls:
        B, rows = len(ls), sum(ns)
        r, keep = rr.rows_of(ls, ns, c.table[b0: b0 + B])
        q = _dev(c.x[r0: r0 + rows, :8].reshape(rows, -1))
        n = m.kvp_workspace_size(kb.KVP_PHASE_STEP, B, rows)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        work.append((r, keep, q, ws, n, range(b0, b0 + B), r0, torch.cuda.Stream(), layer))
        b0, r0 = b0 + B, r0 + rows

    def attend(w, out, st):
        m.kvp_attention(w[8], w[2].data_ptr(), w[0], out.data_ptr(), w[3].data_ptr(), w[4], st.cuda_stream)

    alone = []
    for w in work:
        out = torch.full_like(w[2], float("nan"))
        attend(w, out, torch.cuda.current_stream())
        torch.cuda.synchronize()
        alone.append(out)
        got = out.float().cpu().numpy().reshape(-1, 8, D)
        for b in w[5]:
            rows = slice(int(c.cu[b]) - w[6], int(c.cu[b + 1]) - w[6])
            want, tol = rr.attention(c.x[c.cu[b]: c.cu[b + 1], :8].astype(np.float64), c.cache.values(c.table, b, lens[b] + new[b]),
                                     lens[b], 8, *((3000, 4) if w[8] else (0, 0)))
            assert (np.abs(got[rows] - want) <= tol).all(), b
    outs = [[torch.full_like(w[2], float("nan")) for _ in range(6)] for w in work]
    torch.cuda.synchronize()
    for i in range(6):
        for w, o in zip(work, outs):
            attend(w, o[i], w[7])
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a, x) for x in o)


def test_graphs_share_a_workspace_and_follow_the_lengths():
    """Captured steps (single tokens; chunks) with a page copy in front, on one workspace, replayed in turn and between eager
    calls, with other lengths, pages and inputs in the device arrays each time: outputs and caches of the same eager call."""
    table, n_pages = _scattered(3, 8, 47)
    n_pages += 4
    s = Stack(4, 2, (0, 0, 2), n_pages, 3, seed=47, windows=((0, 0), (50, 3)))
    rng = np.random.default_rng(48)
    s.step(_normal(rng, 140, s.h), [0, 0, 0], [30, 100, 10], table)
    start = {l: [t.clone() for t in d] for l, d in s.dev.items()}
    news = [[1, 1, 1], [40, 3, 29]]
    n = max(s.m.kvp_workspace_size(kb.KVP_PHASE_STEP, 3, sum(t)) for t in news)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    state = []
    for new in news:
        r, keep = rr.rows_of([30, 100, 10], new, table, max_pos=400)
        x = _dev(_normal(rng, sum(new), s.h))
        state.append((r, keep, x, torch.empty_like(x), _i32([-1, -1]), _i32([-1, -1])))

    def run(i):
        r, _, x, y, src, dst = state[i]
        st = torch.cuda.current_stream().cuda_stream
        s.m.kvp_copy_pages(src.data_ptr(), dst.data_ptr(), 2, st)
        s.m.kvp_step(x.data_ptr(), r, y.data_ptr(), ws.data_ptr(), n, st)

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
    graphs = [torch.cuda.CUDAGraph() for _ in news]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            run(i)
    for rep in range(4):
        lens = [[30, 100, 10], [29, 64, 9], [-1, 77, 3], [10, -1, 0]][rep]
        for i, g in enumerate(graphs):
            state[i][2].copy_(_dev(_normal(rng, sum(news[i]), s.h)))
            state[i][1]["len"].copy_(_i32(lens))
            # Sequence 1 gets a copy of its first page, which it then reads.
            other = n_pages - 1 - rep
            state[i][4].copy_(_i32([int(table[1][0]), -1]))
            state[i][5].copy_(_i32([other, -1]))
            new_table = table.copy()
            new_table[1][0] = other
            state[i][1]["pages"].copy_(_i32(new_table))
            want, got = result(lambda: run(i), i), result(g.replay, i)
            assert torch.isfinite(want[0]).all() and torch.equal(want[0], got[0]), (rep, i)
            assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(want[1], got[1])), (rep, i)


def test_pages_shared_by_the_rows_of_one_call():
    """A prefix that several rows of the table name, and a page named twice by windows that see different parts of it."""
    c = Case(8, 2, [200, 200, 200, 70], [1, 4, 1, 2], seed=70)
    c.table[1][:3] = c.table[2][:3] = c.table[0][:3]
    c.table[3][:1] = c.table[0][:1]
    _fill(c)
    rng = np.random.default_rng(71)
    c.cache.put(c.table, 0, 0, _normal(rng, 2, 192, 2, D))
    for w in ((0, 0), (100, 2), (9, 0)):
        _check_attention(c, _attention(c, window=w[0], sinks=w[1]), *w)


def test_profile_counts_the_launches():
    c = Case(4, 2, [300, 20], [1, 1], seed=72)
    _fill(c)
    dev = c.cache.to_device()
    m = rr.model(4, 2, dev, c.cache.n_pages, 2, 64)
    r, keep = rr.rows_of(c.lens, c.new, c.table)
    n = m.kvp_workspace_size(kb.KVP_PHASE_STEP, 2, 2)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    x = _dev(c.x.reshape(2, -1))
    q = torch.empty(2, 4 * D, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    s, d = _i32([int(c.table[0][0])]), _i32([c.cache.n_pages - 1])
    m.kvp_profile_enable(True)
    p = x.data_ptr()
    m.kvp_append(0, p, p + 8 * D, p + 12 * D, 8 * D, r, q.data_ptr(), _stream())
    m.kvp_attention(0, q.data_ptr(), r, out.data_ptr(), ws.data_ptr(), n, _stream())
    m.kvp_copy_pages(s.data_ptr(), d.data_ptr(), 1, _stream())
    got = m.kvp_profile_read()
    assert {k: v[0] for k, v in got.items()} == {"dec_rope": 1, "dec_attn": 1, "page_copy": 1}
    assert all(v[1] > 0 for v in got.values())
