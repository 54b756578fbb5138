"""The books of pages: every page is free or held by as many as the books say, whatever is done; what is shared is copied
before it is written."""
import random

import pytest

torch = pytest.importorskip("torch")

from paper_2506_15745_gb300.sequences import OutOfPages, Sequences  # noqa: E402


def check(books, live, lent=()):
    held = {}
    for s in live:
        pages = books.pages(s)
        assert len(pages) == -(-books.rows(s) // books.page_size) and len(set(pages)) == len(pages)
        for p in pages:
            held[p] = held.get(p, 0) + 1
    for p in lent:
        held[p] = held.get(p, 0) + 1
    assert all(books.holders(p) == held.get(p, 0) for p in range(books.n_pages))
    assert books.free_pages == books.n_pages - len(held)
    assert len(books) == len(live)


def test_growth_by_rows():
    books = Sequences(4, 16)
    s = books.add()
    assert books.rows(s) == 0 and books.pages(s) == [] and books.free_pages == 4
    assert books.extend(s, 0) == [] and books.pages(s) == []
    for n, pages in ((1, 1), (15, 1), (1, 2), (47, 4)):
        assert books.extend(s, n) == []
        assert len(books.pages(s)) == pages
        check(books, [s])
    with pytest.raises(OutOfPages):
        books.extend(s, 1)
    assert books.rows(s) == 64
    books.remove(s)
    check(books, [])
    with pytest.raises(KeyError):
        books.rows(s)


def test_a_fork_copies_the_last_page_when_it_is_written():
    books = Sequences(10, 16)
    a = books.add(40)
    b = books.fork(a)
    c = books.fork(b)
    assert books.pages(a) == books.pages(b) == books.pages(c) and books.free_pages == 7
    last = books.pages(a)[2]
    (source, target), = books.extend(b, 1)
    assert source == last and books.pages(b) == books.pages(a)[:2] + [target]
    assert books.holders(last) == 2 and books.holders(target) == 1
    assert books.extend(b, 1) == []  # its own by now
    check(books, [a, b, c])
    assert len(books.extend(c, 20)) == 1  # and a page behind it
    assert books.extend(a, 1) == []  # the last holder writes in place
    check(books, [a, b, c])


def test_a_full_last_page_is_not_copied():
    books = Sequences(10, 16)
    a = books.add(32)
    b = books.fork(a)
    assert books.extend(b, 5) == [] and len(books.pages(b)) == 3 and books.pages(b)[:2] == books.pages(a)
    check(books, [a, b])


def test_truncation_then_growth_inside_a_shared_page():
    books = Sequences(10, 16)
    a = books.add(64)
    b = books.fork(a)
    books.truncate(b, 20)
    assert books.pages(b) == books.pages(a)[:2]
    (source, target), = books.extend(b, 1)
    assert source == books.pages(a)[1] and target not in books.pages(a)
    check(books, [a, b])
    books.truncate(b, 0)
    assert books.pages(b) == [] and books.extend(b, 1) == []
    with pytest.raises(ValueError, match="rows"):
        books.truncate(b, 2)


def test_compaction_lends_the_old_pages():
    books = Sequences(8, 16)
    a = books.add(80)
    b = books.fork(a)
    old = books.replace(a, 20)
    assert len(old) == 5 and len(books.pages(a)) == 2 and not set(old) & set(books.pages(a))
    check(books, [a, b], old)
    books.release(old)
    check(books, [a, b])
    assert books.pages(b) == old
    with pytest.raises(OutOfPages):
        books.replace(b, 40)
    check(books, [a, b])
    old = books.pages(b)
    books.remove(b)
    with pytest.raises(ValueError, match="nobody"):
        books.release(old)


def test_out_of_pages_changes_nothing():
    books = Sequences(3, 16)
    a = books.add(24)
    b = books.fork(a)
    before = books.pages(b)
    with pytest.raises(OutOfPages):
        books.extend(b, 16)  # a copy of the last page and a page behind it: one too many
    assert books.pages(b) == before and books.rows(b) == 24
    check(books, [a, b])
    with pytest.raises(OutOfPages):
        books.add(17)
    check(books, [a, b])


def test_refusals():
    for bad in ((0, 16), (4, 0)):
        with pytest.raises(ValueError):
            Sequences(*bad)
    books = Sequences(4, 16)
    s = books.add(3)
    for call in (lambda: books.add(-1), lambda: books.extend(s, -1), lambda: books.truncate(s, -1), lambda: books.replace(s, -1),
                 lambda: books.batch([s], [4], device="cpu"), lambda: books.batch([s], [-1], device="cpu"),
                 lambda: books.batch([s], [], device="cpu"), lambda: books.table([books.add(17)], 1)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: books.fork(99), lambda: books.extend(99, 1), lambda: books.remove(99), lambda: books.table([99])):
        with pytest.raises(KeyError):
            call()


def test_tables():
    books = Sequences(8, 16)
    a, b = books.add(33), books.add()
    t = books.table([b, a, a])
    assert t.dtype == torch.int32 and t.tolist() == [[-1] * 3, books.pages(a), books.pages(a)]
    assert books.table([a], 5).tolist() == [books.pages(a) + [-1, -1]]
    assert books.table([]).shape == (0, 1) and books.table([b]).tolist() == [[-1]]


@pytest.mark.parametrize("seed", range(8))
def test_any_order_of_changes(seed):
    rng = random.Random(seed)
    books = Sequences(rng.choice([5, 20, 60]), rng.choice([1, 7, 16]))
    live, lent = [], []
    for _ in range(400):
        op = rng.choice(["add", "fork", "extend", "extend", "extend", "truncate", "replace", "release", "remove"])
        s = rng.choice(live) if live else None
        try:
            if op == "add":
                live.append(books.add(rng.randint(0, 30)))
            elif op == "release" and lent:
                books.release(lent)
                lent = []
            elif s is None or op == "release":
                continue
            elif op == "fork":
                live.append(books.fork(s))
            elif op == "extend":
                n = rng.randint(0, 20)
                before, rows = books.pages(s), books.rows(s)
                copies = books.extend(s, n)
                after = books.pages(s)
                for source, target in copies:  # the page that gets rows, and no other, is replaced
                    at = rows // books.page_size
                    assert before[at] == source and after[at] == target and books.holders(target) == 1
                for i in range(rows // books.page_size, len(after)):
                    if n:
                        assert books.holders(after[i]) == 1  # whatever is written is held by the writer alone
            elif op == "truncate":
                books.truncate(s, rng.randint(0, books.rows(s)))
            elif op == "replace":
                lent += books.replace(s, rng.randint(0, books.rows(s)))
            else:
                books.remove(s)
                live.remove(s)
        except OutOfPages:
            pass
        check(books, live, lent)


def test_pages_are_given_back_once():
    """What replace lent is given back by that lending alone: a second release, or one of pages never lent, takes nobody else's
    pages away, and one bad page among others changes nothing."""
    books = Sequences(8, 16)
    a = books.add(40)
    b = books.fork(a)
    old = books.replace(a, 16)
    with pytest.raises(ValueError, match="lent"):
        books.release(old + [books.pages(a)[0]])
    with pytest.raises(ValueError, match="lent"):
        books.release(old[:1] + old)
    check(books, [a, b], old)
    books.release(iter(old))
    check(books, [a, b])
    with pytest.raises(ValueError, match="lent"):
        books.release(old)
    with pytest.raises(ValueError, match="lent"):
        books.release(books.pages(b))
    check(books, [a, b])
    assert books.pages(b) == old and books.free_pages == 4
    for bad in (-1, 8):
        with pytest.raises(ValueError, match="lent"):
            books.release([bad])
    c = books.add(64)  # all that is free, and nothing of b
    assert not set(books.pages(c)) & set(books.pages(b))
    check(books, [a, b, c])
