"""The books over cache pages (ls_pages_*) against a model that keeps every token's content: whatever is grown, forked, cut
back and packed, with the copies made that the calls ask for, every row reads what it wrote."""
import random

import pytest

from paper_2507_21276_amd import binding as Bd
from paper_2507_21276_amd import sched


class Model:
    """A pool of page contents on the host and, for every row, the tokens it should read."""

    def __init__(self, n_pages, page, rows, per_row):
        self.p, self.page = sched.Pages(n_pages, page, rows, per_row), page
        self.pool = [[None] * page for _ in range(n_pages)]
        self.want = [[] for _ in range(rows)]
        self.stamp = 0

    def copy(self, pairs):
        src, dst = pairs
        assert not set(src) & set(dst) and len(set(dst)) == len(dst)
        for s, d in zip(src, dst):
            self.pool[d] = list(self.pool[s])
        return len(src)

    def write(self, row, at, n):
        n_copies = self.copy(self.p.grow(row, at, at + n))
        ids = self.p.row(row)
        del self.want[row][at:]
        for i in range(at, at + n):
            self.stamp += 1
            self.pool[ids[i // self.page]][i % self.page] = self.stamp
            self.want[row].append(self.stamp)
        return n_copies

    def check(self):
        held = {}
        for row, want in enumerate(self.want):
            ids = self.p.row(row)
            assert len(ids) >= (len(want) + self.page - 1) // self.page and len(set(ids)) == len(ids)
            assert [self.pool[ids[i // self.page]][i % self.page] for i in range(len(want))] == want
            for i in ids:
                held[i] = held.get(i, 0) + 1
        assert self.p.available() == len(self.pool) - len(held)
        return set(held)


def test_a_fork_shares_pages_until_one_row_writes_into_the_last():
    m = Model(10, 8, 3, 6)
    m.write(0, 0, 20)                            # pages 0, 1, 2
    m.p.fork(0, 1, 20)
    m.want[1] = list(m.want[0])
    assert m.p.row(1) == m.p.row(0) == [0, 1, 2] and m.p.available() == 7
    assert m.write(0, 20, 3) == 1                # tokens 16 .. 19 are copied once
    assert m.p.row(0) == [0, 1, 3] and m.p.row(1) == [0, 1, 2]
    assert m.write(1, 20, 6) == 0                # the other row has the page to itself by now
    assert m.p.row(1) == [0, 1, 2, 4]
    m.p.fork(0, 2, 16)
    m.want[2] = m.want[0][:16]
    assert m.write(2, 16, 1) == 0                # the fork ends at a page's end: nothing to copy
    m.check()
    m.p.truncate(0, 0)
    m.want[0] = []
    assert m.p.row(0) == [] and m.p.available() == 10 - 5
    m.check()


def test_pages_that_are_written_anew_are_not_copied():
    m = Model(8, 8, 2, 4)
    m.write(0, 0, 24)
    m.p.fork(0, 1, 24)
    m.want[1] = list(m.want[0])
    assert m.write(1, 12, 12) == 1               # of two shared pages only the first holds tokens that stay
    assert m.p.row(1)[0] == m.p.row(0)[0] and not set(m.p.row(1)[1:]) & set(m.p.row(0))
    m.check()


def test_growing_by_nothing_leaves_shared_pages_shared():
    p = sched.Pages(3, 8, 2, 3)
    assert p.grow(0, 0, 20) == ([], [])
    p.fork(0, 1, 20)
    for at in (0, 5, 16, 20):                    # no token is written, so no page is asked for: there is none left
        assert p.grow(1, at, at) == ([], []) and p.row(1) == p.row(0) == [0, 1, 2]


def test_compaction_fills_the_lowest_pages():
    m = Model(12, 4, 4, 6)
    for row in range(4):
        m.write(row, 0, 12)
    m.p.truncate(0, 0)
    m.p.truncate(2, 5)
    m.want[0], m.want[2] = [], m.want[2][:5]
    m.p.fork(3, 0, 12)
    m.want[0] = list(m.want[3])
    moves = m.p.compact()
    assert m.copy(moves) == len(moves[0]) > 0 and max(moves[1]) < 8 <= min(moves[0])
    assert m.check() == set(range(8)) and m.p.row(0) == m.p.row(3)
    assert m.p.compact() == ([], [])
    m.write(1, 12, 1)
    assert m.p.row(1)[-1] == 8                   # the lowest free page comes first
    m.check()


@pytest.mark.parametrize("seed", range(6))
def test_random_histories(seed):
    rng = random.Random(seed)
    page, rows, per_row = rng.choice([4, 8]), 6, 7
    m = Model(rng.randint(12, 30), page, rows, per_row)
    for _ in range(400):
        row, op = rng.randrange(rows), rng.random()
        n = len(m.want[row])
        if op < 0.5:
            at = rng.randint(max(0, n - 6), n)
            more = rng.randint(0, min(9, per_row * page - at))
            before = [m.p.row(r) for r in range(rows)]
            try:
                m.write(row, at, more)
            except Bd.LsError as e:
                assert e.status == Bd.LS_ENOMEM and [m.p.row(r) for r in range(rows)] == before
        elif op < 0.7:
            cut = rng.randint(0, n)
            m.p.truncate(row, cut)
            m.want[row] = m.want[row][:cut]
        elif op < 0.9:
            to = rng.randrange(rows)
            if m.p.row(to) == [] and to != row:
                upto = rng.randint(0, n)
                m.p.fork(row, to, upto)
                m.want[to] = m.want[row][:upto]
        else:
            m.copy(m.p.compact())
            held = m.check()
            assert held == set(range(len(held)))
        m.check()


def test_refusals():
    lib = Bd.lib()
    h = Bd.C.c_void_p()
    for bad in ((0, 8, 1, 1), (4, 0, 1, 1), (4, 8, 0, 1), (4, 8, 1, -1)):
        assert lib.ls_pages_create(*bad, Bd.C.byref(h)) == Bd.LS_EINVAL
    assert lib.ls_pages_create(4, 8, 1, 1, None) == Bd.LS_EINVAL
    assert lib.ls_pages_available(None) == 0 and lib.ls_pages_row(None, 0, None, None) == Bd.LS_EINVAL
    lib.ls_pages_destroy(None)
    p = sched.Pages(4, 8, 2, 3)
    for call in (lambda: p.row(2), lambda: p.row(-1), lambda: p.grow(0, 0, 25), lambda: p.grow(0, 5, 4), lambda: p.grow(0, -1, 4),
                 lambda: p.fork(0, 0, 0), lambda: p.fork(0, 1, 1), lambda: p.fork(0, 1, -1), lambda: p.truncate(0, -1), lambda: p.truncate(7, 0)):
        with pytest.raises(Bd.LsError) as e:
            call()
        assert e.value.status == Bd.LS_EINVAL
    p.grow(0, 0, 24)
    with pytest.raises(Bd.LsError) as e:
        p.grow(1, 0, 17)
    assert e.value.status == Bd.LS_ENOMEM and p.row(1) == [] and p.available() == 1
    p.fork(0, 1, 0)                               # no tokens, no pages
    with pytest.raises(Bd.LsError):
        p.fork(1, 0, 0)                           # row 0 is in use
