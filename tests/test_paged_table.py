"""Bookkeeping of shared pages and of tokens that are shed, on the host."""
import pytest


@pytest.fixture()
def table():
    from paper_2607_05061_gb300.paged import PageTable
    return PageTable(5, 8, 24, page=16, device="cpu")


def fill(t, s, n):
    new = [0] * len(t.held)
    new[s] = n
    t.grow(new)
    t.advance(new)


def consistent(t):
    """Every page is free or has as many users as there are rows that hold it."""
    held = [p for row in t.pages for p in row]
    assert all(t.users[p] == held.count(p) for p in range(len(t.users)))
    assert sorted(t.free) == [p for p in range(len(t.users)) if t.users[p] == 0]
    for s, row in enumerate(t.pages):
        assert t.dev[s, :len(row)].tolist() == row and (t.dev[s, len(row):] == -1).all()
    assert t.lens.tolist() == t.held and t.pos.tolist() == t.seen


def test_shared_pages(table):
    table.open(0)
    fill(table, 0, 50)
    assert table.share(0, 2, 40) == 32 and table.pages[2] == table.pages[0][:2]
    assert table.share(0, 1, 1000) == 48
    consistent(table)
    fill(table, 2, 20)                              # its own pages from there on
    assert len(set(table.pages[2]) & set(table.pages[0])) == 2
    consistent(table)
    before = len(table.free)
    table.close(0)                                  # the others still read them
    consistent(table)
    assert len(table.free) == before + 1
    table.close(1)
    table.close(2)
    consistent(table)
    assert len(table.free) == 24


def test_a_page_that_is_not_whole_is_not_shared(table):
    table.open(0)
    fill(table, 0, 15)
    assert table.share(0, 1, 15) == 0 and table.held[1] == 0 and table.pages[1] == []
    consistent(table)
    assert table.share(0, 0 + 1, 0) == 0


def test_share_refuses(table):
    table.open(0)
    fill(table, 0, 33)
    for bad in ((0, 0, 16), (3, 1, 16), (0, 1, -1)):
        with pytest.raises(ValueError):
            table.share(*bad)
    table.shrink(20)
    with pytest.raises(ValueError):
        table.share(0, 1, 16)
    table.shrunk()
    with pytest.raises(ValueError):                 # its heads hold different tokens now
        table.share(0, 1, 16)
    consistent(table)


def test_groups(table):
    assert table.groups() == (None, None)
    for s in (0, 3):
        table.open(s)
        fill(table, s, 40)
    assert table.groups() == (None, None)
    table.share(0, 1, 40)                           # place 2 stays idle
    table.share(3, 4, 16)
    groups, prefix = table.groups()
    assert groups.tolist() == [0, 2, 3, 5] and prefix.tolist() == [32, 0, 16]
    table.share(0, 4, 32)                           # beyond a place that begins otherwise
    groups, prefix = table.groups()
    assert groups.tolist() == [0, 2, 5] and prefix.tolist() == [32, 0]
    table.close(3)
    groups, prefix = table.groups()                 # idle places between them do not matter
    assert groups.tolist() == [0, 5] and prefix.tolist() == [32]


def test_groups_do_not_give_up_long_prefixes(table):
    table.open(0)
    fill(table, 0, 100)
    table.share(0, 1, 100)
    table.share(0, 2, 16)
    groups, prefix = table.groups()
    assert groups.tolist() == [0, 2, 5] and prefix.tolist() == [96, 0]


def test_shedding(table):
    table.open(0)
    table.open(3)
    fill(table, 0, 50)
    fill(table, 3, 20)
    table.share(0, 1, 48)
    old = [list(p) for p in table.pages]
    to = table.shrink(33)
    assert tuple(to.shape) == (5, 3)
    rows = to.tolist()
    assert [sum(p >= 0 for p in r) for r in rows] == [3, 3, 0, 2, 0]
    new = [p for r in rows for p in r if p >= 0]
    assert len(set(new)) == 8 and not set(new) & {p for r in old for p in r}
    assert table.pages == old and table.held == [50, 48, -1, 20, -1]
    for call in (lambda: table.grow(1), lambda: table.close(0), lambda: table.open(2), lambda: table.advance(1)):
        with pytest.raises(ValueError):
            call()
    table.shrunk()
    assert table.held == [33, 33, -1, 20, -1] and table.seen == [50, 48, -1, 20, -1]
    consistent(table)
    assert table.groups() == (None, None)
    assert table.positions([2, 1, 4, 0, 0]).tolist() == [50, 51, 48]
    table.grow(1)
    table.advance(1)
    assert table.pos.tolist() == [51, 49, -1, 21, -1]
    consistent(table)
    with pytest.raises(ValueError):
        table.shrunk()


def test_shrink_that_does_not_fit_or_is_asked_again(table):
    table.open(0)
    fill(table, 0, 128)
    table.open(1)
    fill(table, 1, 128)
    free = list(table.free)
    with pytest.raises(ValueError):
        table.shrink(0)
    table.shrink(32)
    table.shrink(16)                                # the first ones come back
    assert len(table.free) == len(free) - 2
    table.shrunk()
    consistent(table)
    fill(table, 0, 112)
    fill(table, 1, 112)
    table.open(2)
    fill(table, 2, 100)
    with pytest.raises(MemoryError):
        table.shrink(96)
    consistent(table)
    table.grow([0, 0, 1, 0, 0])                     # nothing is pending


def test_steps_on_the_device(table):
    table.open(0)
    table.open(4)
    table.advance_lens()
    table.advance_held(1)
    consistent(table)
    assert table.pos.tolist() == [1, -1, -1, -1, 1]
