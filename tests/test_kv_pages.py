"""Pages of requests that share some (CPU: the kernel source run on the host,
against the oracle)."""
import ctypes

import numpy as np
import pytest

from oracle import spec_decode as S
from tests import _hip_host


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return _hip_host.compile_host("pages", tmp_path_factory.mktemp("hip_host"))


def _p(a):
    return ctypes.c_void_p(a.ctypes.data)


class Cache:
    """The kernel's tables and rows beside the oracle's."""

    def __init__(self, lib, B, n_pages, size, width, layers=2, row=64, seed=0):
        rng = np.random.default_rng(seed)
        self.lib, self.size, self.B, self.n_pages, self.row = lib, size, B, n_pages, row
        self.table = np.full((B, width), -1, np.int32)
        self.held, self.ref = np.zeros(B, np.int32), np.zeros(n_pages, np.int32)
        self.rows = [rng.integers(0, 9999, (layers, n_pages, size, row)).astype(np.uint16)
                     for _ in range(2)]
        self.oracle = S.Pages(self.table, self.held, self.ref, size, [x.copy() for x in self.rows])

    def sync(self):
        """Takes over the oracle's tables and rows (after its fork and trim)."""
        o = self.oracle
        self.table[:], self.held[:], self.ref[:] = o.table, o.held, o.ref
        for x, y in zip(self.rows, o.caches):
            x[:] = y

    def reserve(self, lengths, n):
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        T, lengths = int(off[-1]), np.array(lengths, np.int32)
        slots, status = np.full(max(T, 1), 77, np.int32), np.full(self.B, 9, np.int32)
        self.sync()
        self.lib.reserve(_p(self.table), _p(self.held), _p(self.ref), self.n_pages,
                         self.size.bit_length() - 1, self.B, self.table.shape[1], _p(lengths),
                         _p(off), T, _p(slots), _p(status), *map(_p, self.rows),
                         self.rows[0].shape[0], self.row)
        o_slots, o_status = self.oracle.reserve(lengths, off, T)
        o = self.oracle
        assert np.array_equal(status, o_status)
        assert np.array_equal(slots[:T], o_slots)
        for a, b in zip((self.table, self.held, self.ref, *self.rows),
                        (o.table, o.held, o.ref, *o.caches)):
            assert np.array_equal(a, b)
        for p in slots[:T][slots[:T] >= 0] // self.size:
            assert o.ref[p] == 1, "a new row in a page that others hold"
        return off, slots[:T], status

    def tokens(self, b, n):
        """The first n rows of a request, all layers, K and V."""
        pos = np.arange(n)
        at = self.oracle.table[b, pos // self.size], pos % self.size
        return np.stack([c[:, at[0], at[1]] for c in self.oracle.caches])


def test_rows_after_a_rollback_below_a_fork_leave_the_parent_alone(lib):
    c = Cache(lib, 2, 6, 16, 4)
    c.reserve([0, 0], [32, 0])
    lengths = np.array([32, 0], np.int32)
    assert c.oracle.fork(lengths, [0], [1]).tolist() == [1]
    c.oracle.trim([32, 28])
    parent, child = c.tokens(0, 32), c.tokens(1, 28)
    off, slots, status = c.reserve([32, 28], [0, 4])
    assert status.tolist() == [1, 1] and c.oracle.ref.tolist() == [2, 1, 1, 0, 0, 0]
    for x in c.oracle.caches:
        x[:, slots // 16, slots % 16] = 12345
    assert np.array_equal(c.tokens(0, 32), parent)
    assert np.array_equal(c.tokens(1, 28), child)
    assert (c.tokens(1, 32)[:, :, 28:] == 12345).all()


def test_a_rollback_without_trim_and_both_holders_writing(lib):
    """Lengths taken back over several shared pages that are still held; the
    first and the last holder write, with pages for one only, then with more."""
    for n_pages, want in ((3 + 2, [1, 1, 0]), (3 + 4, [1, 1, 1])):
        c = Cache(lib, 3, n_pages, 4, 5)
        c.reserve([0, 0, 0], [12, 0, 0])
        lengths = np.array([12, 0, 0], np.int32)
        assert c.oracle.fork(lengths, [0, 0], [1, 2]).tolist() == [1, 1]
        before = [c.tokens(b, n) for b, n in enumerate((6, 12, 6))]
        _, slots, status = c.reserve([6, 12, 6], [5, 0, 5])
        assert status.tolist() == want
        for b, n in enumerate((6, 12, 6)):
            assert np.array_equal(c.tokens(b, n), before[b])
        _, _, status = c.reserve([6, 12, 6], [5, 0, 5])  # pages of their own: nothing more
        assert status[0] == 1


def test_an_aligned_rollback_shares_no_page_with_new_rows(lib):
    c = Cache(lib, 2, 8, 8, 4)
    c.reserve([0, 0], [24, 0])
    lengths = np.array([24, 0], np.int32)
    c.oracle.fork(lengths, [0], [1])
    before = c.tokens(0, 24)
    _, slots, status = c.reserve([24, 8], [1, 9])  # two shared pages, none of their rows in use
    assert status.tolist() == [1, 1]
    for x in c.oracle.caches:
        x[:, slots // 8, slots % 8] = 4321
    assert np.array_equal(c.tokens(0, 24), before)


@pytest.mark.parametrize("seed", range(5))
@pytest.mark.parametrize("B,size,n_pages,width", [
    (2, 16, 12, 4), (5, 4, 24, 9), (7, 1, 60, 20), (30, 8, 9000, 12), (1100, 2, 2400, 6)])
def test_sequences_with_rollbacks(lib, B, size, n_pages, width, seed):
    """Reserve, fork and rollbacks (trimmed or not) in a seeded order, running
    out of pages: what every request holds stays, whoever writes."""
    rng = np.random.default_rng(seed)
    c = Cache(lib, B, n_pages, size, width, layers=1, seed=seed)
    lengths = np.zeros(B, np.int32)
    for step in range(6):
        n = rng.integers(0, 2 * size + 2, B) * (rng.random(B) < 0.7)
        held = [c.tokens(b, lengths[b]) for b in range(min(B, 30))]
        off, slots, status = c.reserve(lengths, n)
        ok = slots >= 0
        assert len(set(slots[ok])) == ok.sum()
        for x in c.oracle.caches:
            x[:, slots[ok] // size, slots[ok] % size] = 50000 + step
        for b, x in enumerate(held):
            assert np.array_equal(c.tokens(b, lengths[b]), x), (step, b)
        used = [p for r, h in zip(c.oracle.table, c.oracle.held) for p in r[:h]]
        assert np.array_equal(np.bincount(used, minlength=n_pages), c.oracle.ref)
        lengths = (lengths + n * status).astype(np.int32)
        # A third of the requests end and become copies of others, which then
        # go back, most of them below what they share.
        gone = rng.random(B) < 0.34
        lengths = np.where(gone, 0, lengths).astype(np.int32)
        c.oracle.trim(np.where(gone, 0, c.oracle.held * size))
        dst, src = np.flatnonzero(gone)[:1000], np.flatnonzero(~gone)
        if len(src):
            c.oracle.fork(lengths, rng.choice(src, len(dst)).tolist(), dst.tolist())
        back = np.where(rng.random(B) < 0.7, rng.integers(0, 2 * size + 1, B), 0)
        lengths = np.maximum(lengths - back, 0).astype(np.int32)
        if step % 2:
            c.oracle.trim(lengths)


def test_rows_of_no_request_get_no_slots(lib):
    for B, T in ((0, 70), (2, 70)):
        off, slots, status = np.zeros(B + 1, np.int32), np.full(T, 5, np.int32), np.zeros(2, np.int32)
        table, held, refs = np.full((2, 2), -1, np.int32), np.zeros(2, np.int32), np.zeros(4, np.int32)
        rows = np.zeros((1, 4, 16, 64), np.uint16)
        lib.reserve(_p(table), _p(held), _p(refs), 4, 4, B, 2, _p(held), _p(off), T, _p(slots),
                    _p(status), _p(rows), _p(rows), 1, 64)
        assert (slots == -1).all() and (refs == 0).all()


@pytest.mark.parametrize("T", [0, 1, 3, 9])
def test_rows_past_the_slots_change_nothing_about_sharing(lib, T):
    """Fewer slots than rows: those that there are lie in pages of one holder."""
    c = Cache(lib, 2, 8, 4, 5)
    c.reserve([0, 0], [12, 0])
    c.oracle.fork(np.array([12, 0], np.int32), [0], [1])
    c.sync()
    before = c.tokens(0, 12), c.tokens(1, 2)
    lengths, off = np.array([12, 2], np.int32), np.array([0, 0, 10], np.int32)
    slots, status = np.full(max(T, 1), 77, np.int32), np.zeros(2, np.int32)
    lib.reserve(_p(c.table), _p(c.held), _p(c.ref), 8, 2, 2, 5, _p(lengths), _p(off), T, _p(slots),
                _p(status), *map(_p, c.rows), 2, c.row)
    assert status.tolist() == [1, 1] and (slots[T:] == 77).all()
    assert all(c.ref[p] == 1 for p in slots[:T] // 4)
    for x in c.rows:
        x[:, slots[:T] // 4, slots[:T] % 4] = 1
    c.oracle.table, c.oracle.caches = c.table, c.rows
    assert np.array_equal(c.tokens(0, 12), before[0]) and np.array_equal(c.tokens(1, 2), before[1])
