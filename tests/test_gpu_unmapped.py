"""Appends at positions whose table entry is -1, no page, on the GPU: nothing of the pools changes for them, on bf16 and on 8-bit
pages; everything else of the call is as it would be."""
import numpy as np
import pytest
import torch

import lowbit_ref as lr
import rows_ref as rr
import test_gpu_fp8_cache as t8
import test_gpu_rows as t16
from gpu_util import say
from paper_2608_15943_amd import binding as kb
from test_gpu_pages import Stack, _dev, _normal, _scattered

pytestmark = pytest.mark.gpu
KINDS = {"bf16": (rr, t16), "fp8": (lr, t8)}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kb.lib()


def _check(kind, c, gone):
    """c with the entries `gone` [(sequence, entry)] taken out of its table.  Its positions there are appended nowhere."""
    ref, t = KINDS[kind]
    kv = c.kv64()
    lens, new, want, table = [], [], [], []
    for b, (n, T) in enumerate(zip(c.lens, c.new)):
        # A sequence's rows, page by page; those of pages that are there.
        at = n
        while T and at < n + T:
            end = min(n + T, (at // 64 + 1) * 64)
            if (b, at // 64) not in gone:
                lens.append(at), new.append(end - at), want.append(kv[b][:, at - n: end - n]), table.append(c.table[b].copy())
            at = end
    for b, j in gone:
        c.table[b][j] = -1
    after, q_out = t._append(c)
    ref.check_append(c.cache, after, table, lens, new, want)
    t._check_q(c, q_out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("a,g,lens,new,gone", [
    # one row each; a sequence whose page 0 of the pool is another's; every one gone
    (4, 2, [10, 70, 64, 63], [1, 1, 1, 1], [(1, 1), (3, 0)]), (3, 1, [5], [1], [(0, 0)]), (16, 1, [64, 0], [1, 1], [(0, 1), (1, 0)]),
    # rows that go on in the next page, or come from the one before
    (4, 2, [60, 30], [10, 3], [(0, 1)]), (4, 2, [60, 30], [10, 3], [(0, 0)]), (8, 4, [50, 3, 100], [200, 40, 60], [(0, 2), (2, 1)]),
    (2, 2, [0, 0], [64, 65], [(0, 0), (1, 1)]), (4, 2, [13], [300], [(0, j) for j in range(5)])])
def test_append_where_there_is_no_page(kind, a, g, lens, new, gone):
    say(f"[unmapped append] {kind} a={a} g={g} lens={lens} new={new} gone={gone}")
    _check(kind, KINDS[kind][1].Case(a, g, lens, new, seed=7 + len(gone)), gone)


@pytest.mark.parametrize("new", [[1, 1, 1], [3, 5, 70]])
@pytest.mark.parametrize("fp8", [False, True])
def test_step_where_there_is_no_page(new, fp8):
    """A sequence without a page for its rows beside others: it changes no page of the pools, and the others' rows and pages are
    those of a call in which it has its own."""
    say(f"[unmapped step] fp8={fp8} new={new}")
    table, n_pages = _scattered(3, 3, 80)
    s = Stack(4, 2, (0, 0, 2), n_pages, 3, seed=80)
    if fp8:
        s.dev16, s.dev = s.dev, {l: lr.Cache(2, n_pages, l).to_device() for l in s.dev}
        for l, t in s.dev.items():
            s.m.kvp_set_kv_pool_fp8(l, *(x.data_ptr() for x in t), n_pages)
    rng = np.random.default_rng(81)

    def step(x, lens, new, table):
        r, keep = rr.rows_of(lens, new, table, max_pos=150)
        n = s.m.kvp_workspace_size(kb.KVP_PHASE_STEP_FP8 if fp8 else kb.KVP_PHASE_STEP, 3, r.rows)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        y = torch.empty_like(x)
        (s.m.kvp_step_fp8 if fp8 else s.m.kvp_step)(x.data_ptr(), r, y.data_ptr(), ws.data_ptr(), n,
                                                   torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return y.clone(), [t.clone() for d in s.dev.values() for t in d]

    step(_dev(_normal(rng, 90, s.h)), [0, 0, 0], [30, 40, 20], table)
    start = [t.clone() for d in s.dev.values() for t in d]
    x = _dev(_normal(rng, sum(new), s.h))
    want = step(x, [30, 40, 20], new, table)
    for t, u in zip((t for d in s.dev.values() for t in d), start):
        t.copy_(u)
    bad = table.copy()
    bad[2] = -1
    got = step(x, [30, 40, 20], new, bad)
    assert torch.equal(got[0][: new[0] + new[1]], want[0][: new[0] + new[1]])
    for p, q, u in zip(got[1], want[1], start):
        q[:, table[2].tolist()] = u[:, table[2].tolist()]
        assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))


def test_rejected_tokens_give_their_pages_back():
    """Two sequences that propose tokens, accept some and let go of the others' pages, which the other one may get, beside a fork
    of the first; every step as the host's."""
    say("[rejected tokens]")
    pool, stride = 12, 8
    s = Stack(4, 2, (0, 0, 2), pool, 3, seed=85)
    p = kb.Pager(pool, 3, stride)
    rng = np.random.default_rng(86)
    lens, ids = [0, 0], [0, 1]
    news = [[60, 30]] + [[int(rng.integers(1, 70)), int(rng.integers(1, 70))] for _ in range(14)]
    gone = 0
    for i, new in enumerate(news):
        if i == 5:
            p.fork(0, 2, lens[0])
            for l in s.dev:
                s.kv[l, 2] = s.kv[l, 0][:, : lens[0]].copy()
            ids, lens = [0, 1, 2], lens + [lens[0]]
        new = (new + [5])[: len(ids)]
        for b, n, t in zip(ids, lens, new):
            src, dst = p.own(b, n, n + t)
            if src.size:
                a, d = (torch.tensor(np.asarray(z, np.int32)).cuda() for z in (src, dst))
                s.m.kvp_copy_pages(a.data_ptr(), d.data_ptr(), src.size, torch.cuda.current_stream().cuda_stream)
            p.reserve(b, n + t)
        x = _normal(rng, sum(new), s.h)
        want = s.host(x, lens, new, seqs=ids)
        got = s.step(x, lens, new, p.rows(ids))
        assert np.abs(got - want).max() <= 2e-2 * np.abs(want).max(), (i, lens, new)
        keep = [int(rng.integers(0, min(t, 12) + 1)) for t in new]
        free = p.free_pages()
        for j, (b, n, t, k) in enumerate(zip(ids, lens, new, keep)):
            p.trim(b, n + k, 64 * stride)
            lens[j] = n + k
        gone += p.free_pages() - free
    assert gone > 5


@pytest.mark.parametrize("B,a,w4", [(3, 4, None), (20, 4, None), (3, 3, None), (5, 4, 64)])
def test_decode_step_where_there_is_no_page(B, a, w4):
    """The same of kvp_decode_step_paged, whose single tokens go through other kernels: of small batches, of larger ones, of a
    width that no small-batch kernel takes, with 4-bit weights."""
    say(f"[unmapped decode] B={B} a={a} w4={w4}")
    table, n_pages = _scattered(B, 2, 82)
    s = Stack(a, 1, (0, 0, 2), n_pages, B, seed=82, w4=w4)
    rng = np.random.default_rng(83)
    for d in s.dev.values():
        for t in d:
            t.copy_(torch.randn(t.shape, device="cuda"))
    start = [t.clone() for d in s.dev.values() for t in d]
    lens = [(37 * b + 60) % 127 for b in range(B)]
    gone = [0, B - 1]
    n = s.m.kvp_workspace_size(kb.KVP_PHASE_DECODE, B, 1)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    x = _dev(_normal(rng, B, s.h))
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def step(table):
        for t, u in zip((t for d in s.dev.values() for t in d), start):
            t.copy_(u)
        pt = torch.from_numpy(table).cuda()
        y = torch.empty_like(x)
        s.m.kvp_decode_step_paged(x.data_ptr(), dl.data_ptr(), 127, pt.data_ptr(), 2, y.data_ptr(), B, ws.data_ptr(), n,
                                  torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return y, [t.clone() for d in s.dev.values() for t in d]

    want = step(table)
    bad = table.copy()
    for b in gone:
        bad[b, lens[b] // 64] = -1
    got = step(bad)
    rest = [b for b in range(B) if b not in gone]
    assert torch.equal(got[0][rest], want[0][rest])
    for p, q, u in zip(got[1], want[1], start):
        q[:, table[gone].ravel().tolist()] = u[:, table[gone].ravel().tolist()]
        assert torch.equal(p, q)
