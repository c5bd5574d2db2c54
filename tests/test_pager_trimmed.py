"""The page allocator where a trim took pages that somebody asks for again (CPU): rows cut back to the tokens that were
accepted, and forks and rollbacks to positions behind a window."""
import numpy as np
import pytest

from paper_2608_15943_amd import binding as kb


def _code(f, *a):
    with pytest.raises(kb.KvpError) as e:
        f(*a)
    return e.value.code


def _state(p, n):
    return p.rows(list(range(n))).tolist(), p.free_pages()


# ---- own --------------------------------------------------------------------------------------------

def test_own_gives_a_rows_end_that_was_trimmed_its_pages_again():
    p = kb.Pager(8, 2, 6)
    p.reserve(0, 64)
    p.reserve(1, 300)                                   # 1 .. 5
    p.trim(1, 192, 320)                                 # 100 tokens were not accepted
    assert p.rows([1]).tolist() == [[1, 2, 3, -1, -1, -1]] and p.free_pages() == 4
    src, dst = p.own(1, 192, 257)
    assert src.size == dst.size == 0                    # nothing to copy
    row = p.rows([1])[0].tolist()
    assert row[:3] == [1, 2, 3] and row[5] == -1 and p.free_pages() == 2
    assert sorted(row[:5] + [0]) == sorted(set(row[:5] + [0])) and min(row[:5]) >= 0


def test_own_of_a_trimmed_end_stops_at_its_range_and_at_the_rows_end():
    p = kb.Pager(12, 1, 10)
    p.reserve(0, 512)
    p.trim(0, 128, 512)
    p.own(0, 128, 190)
    assert [v >= 0 for v in p.rows([0])[0]] == [True] * 3 + [False] * 7 and p.free_pages() == 9
    assert p.own(0, 190, 2**20)[0].size == 0            # the row's end is at 512
    assert [v >= 0 for v in p.rows([0])[0]] == [True] * 8 + [False] * 2 and p.free_pages() == 4


def test_own_maps_what_was_trimmed_in_front_of_pages_reserved_ahead():
    p = kb.Pager(12, 1, 10)
    p.reserve(0, 600)
    p.trim(0, 192, 320)                                 # 3 and 4; 5 .. 9 were reserved ahead
    p.own(0, 150, 260)
    row = p.rows([0])[0].tolist()
    assert row[:3] + row[5:] == [0, 1, 2, 5, 6, 7, 8, 9] and len(set(row)) == 10 and min(row) >= 0
    p.trim(0, 0, 192)                                   # a window has passed: gone from the beginning on
    p.trim(0, 256, 300)
    assert p.own(0, 0, 64)[0].size == 0 and p.rows([0])[0, 0] == -1
    assert p.own(0, 220, 320)[0].size == 0 and (p.rows([0])[0, 3:] >= 0).all()


def test_own_copies_what_is_shared_and_maps_what_was_trimmed_in_one_call():
    p = kb.Pager(9, 2, 6)
    p.reserve(0, 300)
    p.fork(0, 1, 150)                                   # shares 0, 1, 2
    p.trim(0, 192, 320)
    src, dst = p.own(0, 150, 320)
    row = p.rows([0])[0].tolist()
    assert src.tolist() == [2] and dst.tolist() == [row[2]] and row[:2] == [0, 1] and min(row[:5]) >= 0
    assert p.rows([1]).tolist() == [[0, 1, 2, -1, -1, -1]] and p.free_pages() == 9 - 6
    assert len(set(row[:5] + [2])) == 6


def test_own_of_a_trimmed_end_is_all_or_nothing():
    p = kb.Pager(7, 2, 6)
    p.reserve(0, 300)
    p.fork(0, 1, 150)
    p.trim(0, 192, 320)
    p.reserve(1, 192 + 128)                             # two of the four free pages
    before = _state(p, 2)
    assert before[1] == 2
    assert _code(p.own, 0, 150, 320) == kb.KVP_E_CAPACITY           # one to copy, two to map
    assert _code(p.own, 0, 150, 256, 0) == kb.KVP_E_CAPACITY        # no room for the pair
    assert _state(p, 2) == before
    src, _ = p.own(0, 150, 256)
    assert src.tolist() == [2] and p.free_pages() == 0 and p.rows([0])[0, 4] == -1


def test_own_refuses_positions_behind_ones_that_are_gone():
    """Rows at `from` follow the position in front of it; where that has no page, no page of `from` makes the row whole."""
    p = kb.Pager(20, 2, 16)
    p.reserve(0, 1024)
    p.trim(0, 64, 960)
    p.fork(0, 1, 900)                                   # a fork to a position behind the window: nothing but page 0 is there
    assert p.rows([1]).tolist() == [[0] + [-1] * 15]
    before = _state(p, 2)
    for lo in (900, 896, 128):                          # inside a page that is gone, and on the border of one
        assert _code(p.own, 1, lo, 910 if lo > 800 else 140) == kb.KVP_E_CAPACITY
    assert _code(p.own, 0, 700, 980) == kb.KVP_E_CAPACITY           # a rollback into what was trimmed
    assert _code(p.own, 0, 100, 110) == kb.KVP_E_CAPACITY
    assert _state(p, 2) == before
    p.own(1, 64, 70)                                    # right behind what is there
    assert p.rows([1])[0, 1] >= 0 and p.free_pages() == before[1] - 1
    assert p.own(0, 960, 1024)[0].size == 0             # the window's own pages
    p.trim(0, 0, 1024)
    assert p.own(0, 0, 1)[0].size == 0 and p.rows([0])[0, 0] >= 0   # from the beginning again


# ---- reserve ----------------------------------------------------------------------------------------

def test_reserve_refuses_a_row_whose_end_was_trimmed():
    p = kb.Pager(12, 2, 10)
    p.reserve(0, 64)
    p.reserve(1, 300)
    p.trim(1, 192, 320)
    before = _state(p, 2)
    for n in (193, 256, 300, 320, 321, 500):            # positions from 192 on, with growth and without
        assert not p.try_reserve(1, n)
        assert _code(p.reserve, 1, n) == kb.KVP_E_CAPACITY
    for n in (0, 64, 100, 192):                         # all there
        p.reserve(1, n)
    assert _state(p, 2) == before
    p.own(1, 192, 300)
    p.reserve(1, 300)
    p.reserve(1, 321)
    assert (p.rows([1])[0, :6] >= 0).all()


def test_reserve_refuses_a_fork_to_behind_a_window():
    p = kb.Pager(24, 2, 20)
    p.reserve(0, 1280)
    p.trim(0, 64, 1024)
    p.fork(0, 1, 1000)
    for n in (1000, 1024, 1100):
        assert not p.try_reserve(1, n)
    p.release(1)
    p.fork(0, 1, 1030)                                  # the window's pages: goes on
    p.reserve(1, 1100)
    assert p.own(1, 1030, 1100)[0].size == 1 and (p.rows([1])[0, 16:18] >= 0).all()


def test_reserve_grows_rows_with_a_window():
    for window, sinks in ((1, 0), (64, 3), (130, 0), (200, 70)):
        p = kb.Pager(12, 1, 40)
        n = 0
        for new in [70, 58, 64, 1, 63] + [37] * 40:
            p.reserve(0, n + new)
            p.trim(0, sinks, n - window + 1)            # what the next rows do not see
            row = p.rows([0])[0]
            for t in range(n, n + new):
                j = np.arange(t + 1)
                assert (row[j[(j > t - window) | (j < sinks)] // 64] >= 0).all()
            n += new
        assert n > 12 * 64


# ---- as a server calls them ----------------------------------------------------------------------------

@pytest.mark.parametrize("seed", range(6))
def test_serving_with_rejected_tokens_windows_and_forks(seed):
    """Random steps of sequences with a window: own, reserve, copies, rows written; some are not accepted and their pages
    trimmed, at times a sequence is forked.  Every row written reads, through its sequence's pages, what the sequence wrote at each
    position that it sees; and the calls refuse for want of pages alone."""
    rng = np.random.RandomState(seed)
    pages, seqs, width = [20, 9, 9, 16, 9, 24][seed], 5, 24
    window, sinks = [(10**6, 0), (150, 5), (64, 70), (300, 0), (33, 1), (500, 128)][seed]
    p = kb.Pager(pages, seqs, width)
    pool = np.full((pages, 64), -1)
    said = [[] for _ in range(seqs)]                    # what each sequence wrote
    name = steps = refused = 0
    for _ in range(1000):
        s, op = int(rng.randint(seqs)), rng.rand()
        n = len(said[s])
        if op < 0.75:
            new = int(rng.choice([1, 3, 30, 100]))
            if n + new > 64 * width:
                p.release(s)
                said[s] = []
                continue
            try:
                src, dst = p.own(s, n, n + new)
                pool[dst] = pool[src]
                p.reserve(s, n + new)
            except kb.KvpError as e:
                assert e.code == kb.KVP_E_CAPACITY
                refused += 1
                assert p.free_pages() < new // 64 + 2
                p.release(s)
                said[s] = []
                continue
            row = p.rows([s])[0]
            t = np.arange(n, n + new)
            pool[row[t // 64], t % 64] = name + t - n
            said[s] = said[s] + list(range(name, name + new))
            name += new
            steps += 1
            for at in t:
                j = np.arange(at + 1)
                j = j[(j > at - window) | (j < sinks)]
                assert (row[j // 64] >= 0).all() and (pool[row[j // 64], j % 64] == np.array(said[s])[j]).all()
            if rng.rand() < 0.4:                        # not all of them accepted
                keep = n + int(rng.randint(0, new + 1))
                said[s] = said[s][:keep]
                p.trim(s, keep, 2**31 - 1 if rng.rand() < 0.5 else 64 * (-(-(n + new) // 64)))
            p.trim(s, sinks, len(said[s]) - window + 1)
        elif op < 0.85:
            t = int(rng.randint(seqs))
            if t != s and n:
                p.release(t)
                p.fork(s, t, n)
                said[t] = list(said[s])
        elif op < 0.95:
            src, dst = p.compact(int(rng.randint(1, 8)))
            pool[dst] = pool[src]
        else:
            p.release(s)
            said[s] = []
    assert steps > 300 and refused > 0
