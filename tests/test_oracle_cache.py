"""Pins of the oracle's paged cache: against plain lists of rows, and its own bookkeeping."""
import numpy as np
import pytest

from oracle import cache as OC
from tests import cache_drafts


def rows_of(c, s):
    n = int(c.lens[s])
    return c.gather([s] * n, range(n))[:, 0].tolist()


def check_holders(c):
    held = np.zeros_like(c.refs)
    for s, n in enumerate(c.lens):
        k = -(-int(n) // c.page_rows)
        assert np.all(c.table[s, :k] >= 0) and np.all(c.table[s, k:] == -1)
        assert len(set(c.table[s, :k].tolist())) == k
        np.add.at(held, c.table[s, :k], 1)
    assert np.array_equal(held, c.refs)


@pytest.mark.parametrize("page_rows", [1, 3, 4])
def test_random_runs_against_lists(page_rows):
    rng = np.random.default_rng(page_rows)
    c = OC.Cache(14, page_rows, (1,), 7, 4)
    lists = [[] for _ in range(7)]
    fresh, seen = 1, set()
    for _ in range(300):
        do = max(0, rng.integers(-2, 4))
        if do == 0:
            seq = rng.integers(-1, 8, rng.integers(1, 4)).tolist()
            row0 = np.concatenate([[0], np.cumsum(rng.integers(0, 5, len(seq)))])
            rows = np.arange(fresh, fresh + row0[-1], dtype=np.uint32)[:, None]
            fresh += int(row0[-1])
            status = c.append(seq, rows, row0)
            for i, s in enumerate(seq):
                if status[i] == OC.OK:
                    lists[s] += rows[row0[i]:row0[i + 1], 0].tolist()
        elif do == 1:
            src, dst = rng.integers(-1, 8, 3).tolist(), rng.integers(-1, 8, 3).tolist()
            was = [list(v) for v in lists]
            status = c.fork(src, dst)
            for s, d, st in zip(src, dst, status):
                if st == OC.OK:
                    lists[d] = list(was[s])
        elif do == 2:
            seq, keep = rng.integers(-1, 8, 2).tolist(), rng.integers(-2, 12, 2).tolist()
            status = c.free(seq, keep)
            for s, k, st in zip(seq, keep, status):
                if st == OC.OK:
                    lists[s] = lists[s][: max(0, k)]
        else:
            status = []
            live = c.compact()
            assert np.all(c.refs[:live] > 0) and np.all(c.refs[live:] == 0)
        seen.update(status)
        check_holders(c)
        assert [rows_of(c, s) for s in range(7)] == lists
    assert seen == {OC.OK, OC.BAD_REQUEST, OC.TABLE_FULL, OC.NO_PAGES}


def test_the_last_of_all_holders_keeps_a_shared_page():
    c = OC.Cache(8, 4, (1,), 3, 2)
    c.append([0], np.array([[1], [2]], np.uint32), [0, 2])
    c.fork([0, 0], [1, 2])
    page = c.table[0, 0]
    assert c.append([2, 0, 1], np.array([[3], [4], [5]], np.uint32)) == [OC.OK] * 3
    assert c.table[1, 0] == page and c.refs[page] == 1
    assert [rows_of(c, s) for s in range(3)] == [[1, 2, 4], [1, 2, 5], [1, 2, 3]]


def test_a_row_that_is_not_there_gathers_as_zeros():
    c = OC.Cache(2, 2, (1,), 2, 2)
    c.append([0], np.array([[7]], np.uint32))
    assert c.gather([0, 0, 0, 1, -1, 2], [0, 1, -1, 0, 0, 0])[:, 0].tolist() == [7, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("order", [[0, 1, 2], [0, 2, 1], [2, 1, 0], [1, 0, 2]])
def test_the_longest_of_all_holders_keeps_a_shared_page(order):
    """Holders of 3, 1 and 2 rows on one page: none of the rows that the others copy is written in the call."""
    c = OC.Cache(8, 4, (1,), 3, 2)
    c.append([0], np.array([[10], [11], [12]], np.uint32), [0, 3])
    c.fork([0, 0], [1, 2])
    c.free([1, 2], [1, 2])
    page, before = c.table[0, 0], c.table.copy()
    assert c.append(order, np.array([[100 + s] for s in order], np.uint32)) == [OC.OK] * 3
    assert c.table[0, 0] == page and c.refs[page] == 1
    assert [rows_of(c, s) for s in range(3)] == [[10, 11, 12, 100], [10, 101], [10, 11, 102]]
    assert not cache_drafts.clashes([3, 1, 2], before, c.table, 4, order, [1] * 3)


@pytest.mark.parametrize("page_rows", [3, 4, 5, 8])
def test_drafts_against_lists(page_rows):
    rng = np.random.default_rng(30 + page_rows)
    c = OC.Cache(40, page_rows, (1,), cache_drafts.SEQS, 6)
    lists = [[] for _ in range(cache_drafts.SEQS)]
    fresh, kept, unlike = 1, 0, 0
    for name, *args in cache_drafts.calls(rng, 60, page_rows):
        if name == "append":
            seq, counts = args
            row0 = np.concatenate([[0], np.cumsum(counts)])
            rows = np.arange(fresh, fresh + row0[-1], dtype=np.uint32)[:, None]
            fresh += int(row0[-1])
            lens, table = c.lens.copy(), c.table.copy()
            k, u = cache_drafts.shared_last_pages(lens, table, c.refs, page_rows, seq, counts)
            kept, unlike = kept + k, unlike + u
            assert c.append(seq, rows, row0) == [OC.OK] * len(seq)
            assert not cache_drafts.clashes(lens, table, c.table, page_rows, seq, counts)
            for i, s in enumerate(seq):
                lists[s] += rows[row0[i]:row0[i + 1], 0].tolist()
        elif name == "fork":
            assert c.fork(*args) == [OC.OK] * len(args[0])
            for s, d in zip(*args):
                lists[d] = list(lists[s])
        elif name == "free":
            assert c.free(*args) == [OC.OK] * len(args[0])
            for i, s in enumerate(args[0]):
                lists[s] = lists[s][: args[1][i] if args[1] else 0]
        else:
            c.compact()
        check_holders(c)
        assert [rows_of(c, s) for s in range(cache_drafts.SEQS)] == lists
    assert kept >= 10 and unlike >= 5
