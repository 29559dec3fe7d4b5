"""Page tables of the branching cache on the CPU: every call against a model
that stores each token's content by (page, row) and each sequence's content
as a plain list."""
import random

import pytest

from page_tables import FULL, INVALID, OK, Book


class Model:
    """Sequences as lists of tokens; page contents follow the copies that the
    host code asks for and the tokens written through its tables."""

    def __init__(self, book, shift):
        self.book, self.page = book, 1 << shift
        self.seqs, self.cells, self.next = {}, {}, 0

    def place(self, s, i):
        first, _, pages = self.book.get(s)
        return pages[(first + i) // self.page], (first + i) % self.page

    def copy(self, copies):
        before = dict(self.cells)  # all copies read what was there before the launch
        for src, dst, rows in copies:
            for r in range(rows):
                self.cells[dst, r] = before.get((src, r))

    def write(self, s, n):
        """n new tokens at the end of s, in pages that no other sequence holds."""
        refs = self.book.refs()
        for _ in range(n):
            self.next += 1
            self.seqs[s].append(self.next)
            at = self.place(s, len(self.seqs[s]) - 1)
            assert refs[at[0]] == 1
            self.cells[at] = self.next

    def check(self):
        held = {}
        for s in range(self.book.max_seqs):
            got = self.book.get(s)
            if s not in self.seqs:
                assert got is None
                continue
            first, tokens, pages = got
            want = self.seqs[s]
            assert tokens == len(want) and len(set(pages)) == len(pages)
            assert 0 <= first < self.page and (tokens or not first)
            assert len(pages) == -(-(first + tokens) // self.page)
            assert [self.cells[self.place(s, i)] for i in range(tokens)] == want
            for p in pages:
                held[p] = held.get(p, 0) + 1
        assert self.book.refs() == [held.get(p, 0) for p in range(self.book.n_pages)]
        assert self.book.state()[2] == len(held) and self.book.state()[3] == len(self.seqs)


@pytest.mark.parametrize("seed", range(12))
def test_random_calls_keep_every_sequence_and_refuse_without_a_change(seed):
    rng = random.Random(seed)
    shift = 4
    n_pages, max_seqs = rng.choice([3, 17, 40]), rng.choice([1, 5, 9])
    book = Book(n_pages, shift, max_seqs)
    m = Model(book, shift)
    done = dict.fromkeys(("create", "fork", "extend", "trim", "free", "compact", "refused"), 0)
    for _ in range(400):
        op = rng.choice(["create", "fork", "extend", "extend", "extend", "trim", "free", "compact"])
        before = book.state()
        live = sorted(m.seqs)
        if op == "create":
            status, s = book.create()
            if status == OK:
                assert s == min(set(range(max_seqs)) - set(live))
                m.seqs[s] = []
            else:
                assert status == FULL and len(live) == max_seqs
        elif op == "fork" and live:
            src, n = rng.choice(live), rng.randint(0, 3)
            status, out = book.fork(src, n)
            if status == OK:
                assert out == sorted(set(range(max_seqs)) - set(live))[:n]
                for s in out:
                    m.seqs[s] = list(m.seqs[src])
            else:
                assert status == FULL and n > max_seqs - len(live)
        elif op == "extend" and live:
            seqs = rng.sample(live, rng.randint(1, len(live)))
            tokens = [rng.choice([0, 1, 3, 16, rng.randint(0, 60)]) for _ in seqs]
            status, copies = book.extend(seqs, tokens)
            if status == OK:
                m.copy(copies)
                for s, n in zip(seqs, tokens):
                    m.write(s, n)
            else:
                assert status == FULL
        elif op == "trim" and live:
            s = rng.choice(live)
            have = len(m.seqs[s])
            front = rng.randint(0, have + 1)
            back = rng.randint(0, max(0, have - front) + 1)
            status = book.trim(s, front, back)
            if front + back > have:
                assert status == INVALID
            else:
                assert status == OK
                m.seqs[s] = m.seqs[s][front:have - back]
        elif op == "free" and live:
            seqs = rng.sample(live, rng.randint(1, min(2, len(live))))
            status = book.free(seqs)
            assert status == OK
            for s in seqs:
                del m.seqs[s]
        elif op == "compact":
            status, copies = OK, book.compact()
            live_pages = before[2]
            assert [c[0] for c in copies] == [p for p, r in enumerate(before[1]) if r and p >= live_pages]
            assert [c[1] for c in copies] == [p for p, r in enumerate(before[1][:live_pages]) if not r]
            m.copy(copies)
            assert all(book.refs()[:live_pages]) and not any(book.refs()[live_pages:])
        else:
            continue
        done[op if status == OK else "refused"] += 1
        if status != OK:
            assert book.state() == before
        m.check()
    assert all(v for k, v in done.items() if max_seqs > 1 or k != "fork"), done


def _forked():
    book = Book(20, 4, 6)
    assert book.create() == (OK, 0)
    assert book.extend([0], [21]) == (OK, [])
    assert book.fork(0, 3) == (OK, [1, 2, 3])
    return book


def test_last_page_is_copied_for_all_but_its_last_holder():
    book = _forked()
    # the parent grows first: it too gets a copy while others hold the page; of the
    # four holders the last one writes in place
    assert book.extend([0, 2, 1, 3], [1, 1, 0, 12])[1] == [(1, 2, 5), (1, 3, 5), (1, 4, 5)]
    assert book.extend([1], [1])[1] == []
    assert [book.get(s)[2] for s in range(4)] == [[0, 2], [0, 1], [0, 3], [0, 4, 5]]


def test_whole_pages_are_never_copied():
    book = Book(20, 4, 6)
    book.create()
    book.extend([0], [32])
    book.fork(0, 2)
    assert book.extend([1, 2], [40, 1]) == (OK, [])
    assert [book.get(s)[2] for s in (1, 2)] == [[0, 1, 2, 3, 4], [0, 1, 5]]


def test_extend_counts_the_copies_it_needs():
    # three pages free: three of the four holders copy, nothing is left to grow into
    book = Book(5, 4, 6)
    book.create()
    book.extend([0], [21])
    book.fork(0, 3)
    before = book.state()
    assert book.extend([0, 1, 2, 3], [1, 1, 1, 12])[0] == FULL and book.state() == before
    assert book.extend([0, 1, 2, 3], [1, 1, 1, 11])[1] == [(1, 2, 5), (1, 3, 5), (1, 4, 5)]
    assert book.extend([3], [1])[0] == FULL


@pytest.mark.parametrize("call", [
    lambda b: b.fork(4, 1)[0], lambda b: b.fork(-1, 1)[0], lambda b: b.fork(6, 1)[0], lambda b: b.fork(0, -1)[0],
    lambda b: b.extend([4], [1])[0], lambda b: b.extend([0, 0], [1, 1])[0], lambda b: b.extend([0], [-1])[0],
    lambda b: b.extend([0, 99], [1, 1])[0], lambda b: b.trim(5, 0, 0), lambda b: b.trim(0, 22, 0),
    lambda b: b.trim(0, 11, 11), lambda b: b.trim(0, -1, 0), lambda b: b.trim(0, 0, -1), lambda b: b.trim(0, 2**31 - 1, 2**31 - 1),
    lambda b: b.free([4]), lambda b: b.free([1, 1]), lambda b: b.free([-1]),
])
def test_invalid_calls_change_nothing(call):
    book = _forked()
    before = book.state()
    assert call(book) == INVALID
    assert book.state() == before


def test_full_pool_and_huge_lengths():
    book = _forked()
    before = book.state()
    for seqs, tokens in (([1], [2**31 - 1]), ([0, 1], [2**31 - 1, 2**31 - 1]), ([1], [20 * 16])):
        assert book.extend(seqs, tokens)[0] == FULL
        assert book.state() == before
    assert book.fork(0, 3)[0] == FULL and book.state() == before
    assert book.fork(0, 2) == (OK, [4, 5])
    assert book.create()[0] == FULL


def test_versions_change_with_the_table_alone():
    book = _forked()
    v = [book.version(s) for s in range(4)]
    assert len(set(v)) == 4
    book.fork(0, 1)
    book.extend([0, 1], [0, 1])
    assert [book.version(s) == v[s] for s in range(4)] == [True, False, True, True]
    book.trim(2, 0, 0)
    book.free([3])
    assert book.version(2) == v[2]
    book.compact()  # sequence 3's page was shared: nothing moves
    assert book.version(0) == v[0]
    assert book.create() == (OK, 3) and book.version(3) != v[3]
    book.free([0])
    book.extend([2], [100])
    book.free([1, 4])
    moved = book.compact()
    assert moved and book.version(2) != v[2]


def test_front_trim_keeps_the_place_in_the_page():
    book = Book(8, 4, 2)
    book.create()
    book.extend([0], [50])
    assert book.trim(0, 5, 0) == OK and book.get(0) == (5, 45, [0, 1, 2, 3])
    assert book.trim(0, 11, 0) == OK and book.get(0) == (0, 34, [1, 2, 3])
    assert book.trim(0, 33, 0) == OK and book.get(0) == (1, 1, [3])
    assert book.trim(0, 0, 1) == OK and book.get(0) == (0, 0, [])
    assert book.extend([0], [1]) == (OK, []) and book.get(0) == (0, 1, [0])
