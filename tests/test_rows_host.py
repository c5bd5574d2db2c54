"""Host side of the operators on bf16 pages (CPU): the page allocator's sharing, the refusals, the workspace, and the 64-bit
references that the GPU tests use."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest

import rows_ref as rr
from paper_2608_15943_amd import binding as kb

P = 4096          # a non-null, aligned address that no refused call reads


def _model(L=2, a=4, g=2, dtype=kb.KVP_DTYPE_BF16, tau=(0, 0), max_batch=4, max_seq=256):
    return kb.Model(L, a * 128, a, g, 128, dtype, list(tau), max_batch=max_batch, max_seq=max_seq, kv_capacity=max_seq)


def _rows(**kw):
    d = dict(cu=P, len=P, pages=P, pages_stride=4, B=2, rows=6, max_new=4, max_pos=200)
    d.update(kw)
    return kb.kvp_rows(**d)


def _code(f, *a):
    with pytest.raises(kb.KvpError) as e:
        f(*a)
    return e.value.code


# ---- the page allocator ----------------------------------------------------------------------------

def test_fork_shares_pages_until_one_of_the_sequences_owns_them():
    p = kb.Pager(10, 4, 4)
    p.reserve(0, 150)                                   # 0, 1, 2
    p.fork(0, 1, 130)
    assert p.rows([0, 1]).tolist() == [[0, 1, 2, -1]] * 2 and p.free_pages() == 7
    p.fork(1, 2, 64)
    assert p.rows([2]).tolist() == [[0, -1, -1, -1]] and p.free_pages() == 7
    src, dst = p.own(1, 130, 131)                       # appends at 130: page 2 becomes its own
    assert src.tolist() == [2] and dst.tolist() == [3] and p.rows([1]).tolist() == [[0, 1, 3, -1]]
    assert p.own(0, 150, 151)[0].size == 0              # sequence 0 is alone on page 2 now
    src, dst = p.own(0, 0, 192)                         # a rollback to the beginning
    assert src.tolist() == [0, 1] and dst.tolist() == [4, 5] and p.rows([0]).tolist() == [[4, 5, 2, -1]]
    assert p.rows([1, 2]).tolist() == [[0, 1, 3, -1], [0, -1, -1, -1]]
    p.release(1)                                        # page 0 is sequence 2's still
    assert p.free_pages() == 6
    p.release(2)
    assert p.free_pages() == 7
    p.reserve(3, 64)
    assert p.rows([3])[0, 0] == 0                       # released last, handed out first


def test_own_is_all_or_nothing_and_leaves_out_what_has_no_page():
    p = kb.Pager(4, 3, 8)
    p.reserve(0, 192)
    p.fork(0, 1, 192)
    assert _code(p.own, 1, 0, 192) == kb.KVP_E_CAPACITY             # three pages needed, one free
    assert _code(p.own, 1, 64, 128, 0) == kb.KVP_E_CAPACITY         # no room for the pair
    assert p.rows([0, 1]).tolist() == [[0, 1, 2] + [-1] * 5] * 2 and p.free_pages() == 1
    assert p.own(1, 192, 512)[0].size == 0 and p.own(1, 70, 70)[0].size == 0
    assert p.own(1, 127, 128)[0].tolist() == [1]
    p.trim(0, 0, 64)
    assert p.own(0, 0, 64)[0].size == 0                             # a hole


def test_trim_lets_go_of_whole_pages_behind_a_window():
    p = kb.Pager(20, 2, 16)
    p.reserve(0, 1000)
    assert p.free_pages() == 4
    window, sinks, at = 300, 4, 1000
    p.trim(0, sinks, at - window + 1)                   # positions 4 .. 700: pages 1 .. 9 whole
    row = p.rows([0])[0]
    assert (row[1:10] == -1).all() and row[0] == 0 and (row[10:] >= 0).all() and p.free_pages() == 13
    for t in range(at, 1024):
        see = rr.sees(t, np.arange(t + 1), window, sinks)
        assert (row[np.flatnonzero(see) // 64] >= 0).all()
    p.trim(0, sinks, at - window + 1)                   # again: nothing left to let go of
    assert p.free_pages() == 13
    p.reserve(0, 1024)
    assert p.rows([0])[0, 15] == row[15]                # the row's end stayed
    p.trim(0, 640, 639 + 1)
    p.trim(0, 0, 2**31 - 1)
    assert p.free_pages() == 20 and (p.rows([0]) == -1).all()
    p.release(0)
    assert p.free_pages() == 20


def test_fork_of_a_row_with_holes_and_release_in_any_order():
    p = kb.Pager(8, 3, 6)
    p.reserve(0, 384)
    p.trim(0, 64, 256)
    p.fork(0, 1, 384)
    assert p.rows([0]).tolist() == p.rows([1]).tolist() == [[0, -1, -1, -1, 4, 5]]
    p.release(0)
    assert p.free_pages() == 5
    p.release(1)
    assert p.free_pages() == 8


def test_compact_brings_held_pages_to_the_front():
    p = kb.Pager(12, 4, 4)
    for s in range(3):
        p.reserve(s, 256)                               # 0-3, 4-7, 8-11
    p.fork(2, 3, 128)
    p.release(0)
    before = p.rows([1, 2, 3])
    src, dst = p.compact(1)
    assert src.tolist() == [11] and dst.tolist() == [0]
    moves = [(src, dst)]
    while True:
        src, dst = p.compact(2)
        moves.append((src, dst))
        if src.size < 2:
            break
    at = {i: i for i in range(12)}
    for src, dst in moves:
        assert not set(src.tolist()) & set(dst.tolist())
        for x, y in zip(src.tolist(), dst.tolist()):
            at = {k: y if v == x else v for k, v in at.items()}
    after = p.rows([1, 2, 3])
    assert after.max() == 7 and p.free_pages() == 4
    assert (after == np.vectorize(lambda x: at[x] if x >= 0 else -1)(before)).all()
    assert after[1, :2].tolist() == after[2, :2].tolist()           # shared pages moved once
    p.reserve(0, 64)
    assert p.rows([0])[0, 0] == 8                       # lowest first


def test_pager_random_operations_against_a_model():
    """Every page's contents followed by name: what a sequence reads through its row is what it wrote or forked."""
    rng = np.random.RandomState(5)
    n_pages, seqs, width = 60, 7, 12
    p = kb.Pager(n_pages, seqs, width)
    pool = [None] * n_pages
    want = [[] for _ in range(seqs)]
    name = 0
    for _ in range(3000):
        s, op = int(rng.randint(seqs)), rng.rand()
        if op < 0.30:
            n = int(rng.randint(0, width * 64 + 1))
            held = len(want[s])
            if p.try_reserve(s, n):
                row = p.rows([s])[0]
                for j in range(held, (n + 63) // 64):
                    name += 1
                    pool[row[j]] = name
                    want[s].append(name)
        elif op < 0.40:
            p.release(s)
            want[s] = []
        elif op < 0.60:
            t = int(rng.randint(seqs))
            n = int(rng.randint(0, width * 64 + 1))
            legal = t != s and not want[t] and (n + 63) // 64 <= len(want[s])
            if legal:
                p.fork(s, t, n)
                want[t] = want[s][: (n + 63) // 64]
            else:
                assert _code(p.fork, s, t, n) in (kb.KVP_E_INVALID_ARG, kb.KVP_E_STATE, kb.KVP_E_CAPACITY)
        elif op < 0.80 and want[s]:
            lo = int(rng.randint(0, 64 * len(want[s])))
            hi = lo + int(rng.randint(1, 200))
            try:
                src, dst = p.own(s, lo, hi)
            except kb.KvpError as e:
                assert e.code == kb.KVP_E_CAPACITY
                continue
            for x, y in zip(src, dst):
                pool[y] = pool[x]
            row = p.rows([s])[0]
            for j in range(lo // 64, min((hi + 63) // 64, len(want[s]))):      # writes there
                if row[j] >= 0:
                    name += 1
                    pool[row[j]] = want[s][j] = name
        elif op < 0.90:
            lo = int(rng.randint(0, 64 * width))
            hi = lo + int(rng.randint(0, 400))
            p.trim(s, lo, hi)
            for j in range((lo + 63) // 64, min(hi // 64, len(want[s]))):
                want[s][j] = None
        else:
            src, dst = p.compact(int(rng.randint(0, 6)))
            new = [pool[x] for x in src]
            for y, v in zip(dst, new):
                pool[y] = v
        tab = p.rows(list(range(seqs)))
        held = set(tab[tab >= 0].tolist())
        assert len(held) == n_pages - p.free_pages()
        for t in range(seqs):
            assert (tab[t, len(want[t]):] == -1).all()
            for j, v in enumerate(want[t]):
                assert (tab[t, j] < 0) == (v is None) and (v is None or pool[tab[t, j]] == v), (t, j)


def test_pager_refusals():
    p = kb.Pager(8, 2, 4)
    p.reserve(0, 128)
    for args in ((0, 0, 64), (-1, 1, 64), (0, 2, 64), (0, 1, -1)):
        assert _code(p.fork, *args) == kb.KVP_E_INVALID_ARG
    assert _code(p.fork, 0, 1, 129) == kb.KVP_E_CAPACITY
    p.reserve(1, 1)
    assert _code(p.fork, 0, 1, 64) == kb.KVP_E_STATE
    for args in ((2, 0, 64, 4), (0, -1, 64, 4), (0, 64, 63, 4), (0, 0, 64, -1)):
        n = C.c_int(7)
        buf = (C.c_int32 * 4)()
        assert kb.lib().kvp_pager_own(p.p, args[0], args[1], args[2], buf, buf, args[3], C.byref(n)) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_pager_own(p.p, 0, 0, 64, None, None, 1, C.byref(C.c_int())) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_pager_own(p.p, 0, 0, 64, None, None, 0, None) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_pager_own(p.p, 0, 0, 64, None, None, 0, C.byref(C.c_int())) == kb.KVP_OK      # nothing shared
    for args in ((2, 0, 64), (0, -1, 64)):
        assert _code(p.trim, *args) == kb.KVP_E_INVALID_ARG
    before = p.rows([0]).tolist()
    p.trim(0, 3, -200)                                  # no position yet behind the window
    p.trim(0, 64, 64)
    assert p.rows([0]).tolist() == before
    assert kb.lib().kvp_pager_compact(p.p, None, None, 1, C.byref(C.c_int())) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_pager_compact(p.p, None, None, 0, None) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_pager_compact(None, None, None, 0, C.byref(C.c_int())) == kb.KVP_E_INVALID_ARG
    for f in ("kvp_pager_fork", "kvp_pager_trim"):
        assert getattr(kb.lib(), f)(None, 0, 1, 1) == kb.KVP_E_INVALID_ARG


def test_pager_that_no_memory_holds_is_refused():
    """In a process of its own, whose address space is limited."""
    code = ("import resource\n"
            "from paper_2608_15943_amd import binding as kb\n"
            "kb.lib()\n"
            "n = int(open('/proc/self/statm').read().split()[0]) * resource.getpagesize() + (1 << 30)\n"
            "resource.setrlimit(resource.RLIMIT_AS, (n, n))\n"
            "try:\n"
            "    kb.Pager(2**31 - 1, 1, 1)\n"
            "except kb.KvpError as e:\n"
            "    assert e.code == kb.KVP_E_CAPACITY, e\n"
            "    print('refused')\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=root, timeout=120)
    assert r.stdout.strip() == "refused", r.stdout + r.stderr


# ---- refusals ---------------------------------------------------------------------------------------

ROWS = [(dict(len=0), kb.KVP_E_INVALID_ARG), (dict(pages=0), kb.KVP_E_INVALID_ARG),
        (dict(pages_stride=0), kb.KVP_E_INVALID_ARG), (dict(pages_stride=1 << 30), kb.KVP_E_INVALID_ARG),
        (dict(B=0), kb.KVP_E_INVALID_ARG), (dict(rows=0), kb.KVP_E_INVALID_ARG), (dict(max_new=0), kb.KVP_E_INVALID_ARG),
        (dict(max_pos=-1), kb.KVP_E_INVALID_ARG), (dict(cu=0), kb.KVP_E_INVALID_ARG),
        (dict(cu=0, rows=2, max_new=2), kb.KVP_E_INVALID_ARG), (dict(B=5), kb.KVP_E_CAPACITY),
        (dict(max_new=257), kb.KVP_E_CAPACITY), (dict(rows=4 * 256 + 1), kb.KVP_E_CAPACITY),
        (dict(max_pos=256), kb.KVP_E_CAPACITY), (dict(max_pos=2**31 - 1), kb.KVP_E_CAPACITY)]


@pytest.mark.parametrize("kw,code", ROWS)
def test_row_refusals(kw, code):
    m = _model()
    m.kvp_set_kv_pool(0, P, P, 3)
    r = _rows(**kw)
    assert _code(m.kvp_append, 0, P, P, P, 1024, r, P + 16) == code
    assert _code(m.kvp_attention, 0, P, r, P + 16, P, 1 << 40) == code
    assert _code(m.kvp_step, P, r, P + 16, P, 1 << 40) == code


def test_append_refusals():
    m, r = _model(), _rows()
    assert _code(m.kvp_append, 0, P, P, P, 1024, r, P) == kb.KVP_E_STATE        # no pools yet
    m.kvp_set_kv_pool_fp8(0, P, P, P, 3)
    assert _code(m.kvp_append, 0, P, P, P, 1024, r, P) == kb.KVP_E_STATE        # 8-bit ones are others
    m.kvp_set_kv_pool(0, P, P, 3)
    for args in ((2, P, P, P, 1024, r, P + 16), (-1, P, P, P, 1024, r, P + 16), (0, P, P, P, 1024, r, 0), (0, 0, P, P, 1024, r, P),
                 (0, P, P, 0, 1024, r, P + 16), (0, P, 0, P, 1024, r, P + 16), (0, 0, 0, 0, 1024, r, 0),
                 (1, P, P, P, 1024, r, P + 16), (0, P, P, P, 1020, r, P + 16), (0, P, P, P, 504, r, P + 16),
                 (0, 0, P, P, 248, r, 0), (0, P + 2, P, P, 1024, r, P + 16), (0, P, P + 2, P, 1024, r, P + 16),
                 (0, P, P, P + 2, 1024, r, P + 16), (0, P, P, P, 1024, r, P + 2), (0, P, P, P, 1024, r, P)):
        assert _code(m.kvp_append, *args) == kb.KVP_E_INVALID_ARG, args
    assert kb.lib().kvp_append(None, 0, P, P, P, 1024, C.byref(r), P, None) == kb.KVP_E_INVALID_ARG
    assert kb.lib().kvp_append(m.ctx, 0, P, P, P, 1024, None, P, None) == kb.KVP_E_INVALID_ARG
    f = kb.Model(1, 128, 1, 1, 128, kb.KVP_DTYPE_FP32, [0], max_batch=1, max_seq=4, kv_capacity=4)
    assert _code(f.kvp_append, 0, P, P, P, 128, _rows(), P) == kb.KVP_E_SHAPE
    assert _code(f.kvp_workspace_size, kb.KVP_PHASE_STEP, 1, 1) == kb.KVP_E_SHAPE


def test_attention_and_step_refusals():
    m, r = _model(), _rows()
    n = m.kvp_workspace_size(kb.KVP_PHASE_STEP, 2, 6)
    assert _code(m.kvp_attention, 0, P, r, P + 16, P, n) == kb.KVP_E_STATE
    assert _code(m.kvp_step, P, r, P + 16, P, n) == kb.KVP_E_STATE
    m.kvp_set_kv_pool(0, P, P, 3)
    assert _code(m.kvp_step, P, r, P + 16, P, n) == kb.KVP_E_STATE                # no weights
    for args in ((0, 0, r, P), (0, P, r, 0), (0, P, r, P), (0, P + 2, r, P + 16), (0, P, r, P + 2), (2, P, r, P + 16)):
        assert _code(m.kvp_attention, *args, P, n) == kb.KVP_E_INVALID_ARG, args
    for args in ((0, r, P), (P, r, 0), (P, r, P), (P + 2, r, P + 16), (P, r, P + 2)):
        assert _code(m.kvp_step, *args, P, n) == kb.KVP_E_INVALID_ARG, args
    for ws, k in ((0, n), (P, n - 1), (P + 8, n)):
        assert _code(m.kvp_attention, 0, P, r, P + 16, ws, k) == kb.KVP_E_WORKSPACE
        assert _code(m.kvp_step, P, r, P + 16, ws, k) == kb.KVP_E_WORKSPACE
    assert _code(m.kvp_workspace_size, kb.KVP_PHASE_STEP, 5, 6) == kb.KVP_E_CAPACITY
    assert _code(m.kvp_workspace_size, kb.KVP_PHASE_STEP, 4, 1025) == kb.KVP_E_CAPACITY
    assert _code(m.kvp_workspace_size, kb.KVP_PHASE_STEP, 4, 0) == kb.KVP_E_INVALID_ARG
    assert _code(m.kvp_workspace_size, 5, 4, 6) == kb.KVP_E_INVALID_ARG


def test_step_workspace_never_shrinks():
    m = _model(L=1, a=32, g=8, tau=(0,), max_batch=64, max_seq=4096)
    last = 0
    for B, rows in ((1, 1), (1, 2), (2, 16), (2, 63), (4, 64), (4, 65), (4, 66), (8, 200), (64, 2000), (64, 64 * 4096)):
        n = m.kvp_workspace_size(kb.KVP_PHASE_STEP, B, rows)
        assert n >= last, (B, rows)
        last = n


def test_window_refusals():
    m = _model()
    for args in ((2, 4, 0), (-1, 4, 0), (0, -1, 0), (0, 4, -1), (0, 0, 4)):
        assert _code(m.kvp_set_layer_window, *args) == kb.KVP_E_INVALID_ARG, args
    assert kb.lib().kvp_set_layer_window(None, 0, 4, 0) == kb.KVP_E_INVALID_ARG
    f = kb.Model(1, 128, 1, 1, 128, kb.KVP_DTYPE_FP32, [0], max_batch=1, max_seq=4, kv_capacity=4)
    assert _code(f.kvp_set_layer_window, 0, 4, 0) == kb.KVP_E_SHAPE
    m.kvp_set_layer_window(0, 2**31 - 1, 2**31 - 1)
    m.kvp_set_layer_window(0, 0, 0)


def test_calls_that_attend_to_everything_refuse_a_layer_with_a_window():
    """Each gets as far as its check of the layers' state; without a window the fault that it finds next is another."""
    m, r = _model(), _rows()
    for l, kv in ((0, P), (1, 0)):
        m.kvp_set_layer(l, P, kv, kv, P)
        m.kvp_set_layer_grads(l, P, kv, kv, P)
    m.kvp_set_kv_slot(0, P, P)
    m.kvp_set_kv_pool(0, P, P, 3)
    m.kvp_set_kv_pool_fp8(0, P, P, P, 3)
    big, x, y = 1 << 40, P, P + 16
    calls = [(m.kvp_prefill, x, y, 2, 64, P, big), (m.kvp_prefill_paged, x, y, 2, 64, P, 4, P, big),
             (m.kvp_layer_forward, 1, x, 0, y, 2, 64, P, big), (m.kvp_decode_step, x, P, 10, y, 2, P, big),
             (m.kvp_decode_step_paged, x, P, 10, P, 4, y, 2, P, big),
             (m.kvp_train_forward, x, y, 2, 64, P, big, P, big),
             (m.kvp_backward, x, P + 32, y, 2, 64, P, big, P, big), (m.kvp_attention_fp8, 1, x, r, y, P, big),
             (m.kvp_step_fp8, x, r, y, P, big)]
    m.kvp_set_layer_window(1, 16, 2)
    for f, *args in calls:
        assert _code(f, *args) == kb.KVP_E_STATE
        assert "window" in kb.lib().kvp_last_error().decode()


def test_copy_refusals():
    m = _model()
    for f in (m.kvp_copy_pages, m.kvp_copy_pages_fp8):
        assert _code(f, P, P, 1) == kb.KVP_E_STATE              # no pools
    m.kvp_set_kv_pool(0, P, P, 3)
    assert _code(m.kvp_copy_pages_fp8, P, P, 1) == kb.KVP_E_STATE
    m.kvp_set_kv_pool_fp8(0, P, P, P, 3)
    for f in (m.kvp_copy_pages, m.kvp_copy_pages_fp8):
        for args in ((0, P, 1), (P, 0, 1), (P, P, -1)):
            assert _code(f, *args) == kb.KVP_E_INVALID_ARG
        f(0, 0, 0)                                              # nothing to do
    assert kb.lib().kvp_copy_pages(None, P, P, 1, None) == kb.KVP_E_INVALID_ARG
    f = kb.Model(1, 128, 1, 1, 128, kb.KVP_DTYPE_FP32, [0], max_batch=1, max_seq=4, kv_capacity=4)
    assert _code(f.kvp_copy_pages, P, P, 1) == kb.KVP_E_SHAPE


# ---- the references --------------------------------------------------------------------------------

def test_reference_cache_reads_back_what_it_holds():
    rng = np.random.default_rng(0)
    table, n_pages = rr.scattered([3, 2], 3, 2, 1)
    c = rr.Cache(2, n_pages, 3)
    kv = rr.bf16(rng.standard_normal((2, 150, 2, rr.D)))
    c.put(table, 0, 0, kv[:, :100])
    c.put(table, 0, 100, kv[:, 100:])
    assert np.array_equal(c.values(table, 0, 150), kv.astype(np.float64))
    assert not np.isfinite(c.values(table, 1, 1)).all()


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (5, 0), (5, 4), (64, 1), (100, 100)])
def test_reference_attention_is_a_softmax_over_what_a_row_sees(window, sinks):
    """Row by row, over the visible positions alone."""
    rng = np.random.default_rng(1)
    n, T, a, g = 30, 6, 4, 2
    q, kv = rng.standard_normal((T, a, rr.D)), rng.standard_normal((2, n + T, g, rr.D))
    out, tol = rr.attention(q, kv, n, a, window, sinks)
    for t in range(T):
        p = n + t
        seen = [j for j in range(p + 1) if not window or j > p - window or j < sinks]
        for h in range(a):
            s = np.array([kv[0, j, h // 2] @ q[t, h] for j in seen]) / np.sqrt(rr.D)
            w = np.exp(s - s.max())
            w /= w.sum()
            want = sum(x * kv[1, j, h // 2] for x, j in zip(w, seen))
            assert np.allclose(out[t, h], want, rtol=1e-12, atol=1e-12)
            dev = sum(x * np.abs(kv[1, j, h // 2] - want) for x, j in zip(w, seen))
            assert (tol[t, h] >= dev / 255 + 2.0**-8 * np.abs(want) - 1e-12).all()
