"""Groups of a page table against all ways to cut its places into runs (no GPU)."""
import random

import pytest

from paper_2607_05061_gb300.paged import PageTable


def fill(table, s, tokens):
    new = [tokens if i == s else 0 for i in range(len(table.held))]
    table.grow(new)
    table.advance(new)


def saved(table, runs):
    """Reads of pages that runs of places save."""
    total = 0
    for a, b in runs:
        whole = [table.pages[s][:table.held[s] // table.page] for s in range(a, b) if table.held[s] >= 0]
        k = 0
        while whole and all(len(w) > k and w[k] == whole[0][k] for w in whole):
            k += 1
        total += max(len(whole) - 1, 0) * k
    return total


def most(table):
    n = len(table.held)
    return max(saved(table, [(a, b) for a, b in zip([0] + cut, cut + [n])])
               for cut in ([i + 1 for i in range(n - 1) if mask >> i & 1] for mask in range(1 << (n - 1))))


def test_a_short_prefix_does_not_swallow_a_long_one():
    """One page in common with the first place, many among the others: in whichever order they come."""
    for order in ([0, 1, 2, 3, 4], [4, 3, 2, 1, 0], [1, 2, 0, 3, 4]):
        table = PageTable(5, 16, 60, page=16, device="cpu")
        for s in order[:1]:
            table.open(s)
            fill(table, s, 16)
        table.share(order[0], order[1], 16)
        fill(table, order[1], 160)
        for s in order[2:]:
            table.share(order[1], s, 176)
        groups, prefix = table.groups()
        first, p = groups.tolist(), prefix.tolist()
        assert saved(table, list(zip(first, first[1:]))) == most(table) >= 20
        assert 176 in p


@pytest.mark.parametrize("seed", range(40))
def test_groups_save_the_most(seed):
    r = random.Random(seed)
    n = r.randint(1, 9)
    table = PageTable(n, 12, 12 * n, page=16, device="cpu")
    for s in r.sample(range(n), n):
        kind = r.random()
        others = [t for t in range(n) if t != s and table.held[t] >= 0]
        if kind < 0.7 and others:
            t = r.choice(others)
            table.share(t, s, r.randint(0, table.held[t]))
        elif kind < 0.85:
            table.open(s)
        else:
            continue
        fill(table, s, r.randint(0, 12 * 16 - table.held[s]))
    groups, prefix = table.groups()
    if groups is None:
        assert most(table) == 0
        return
    first, p = groups.tolist(), prefix.tolist()
    assert first[0] == 0 and first[-1] == n and first == sorted(set(first)) and len(p) == len(first) - 1
    for a, b, k in zip(first, first[1:], p):
        assert k % 16 == 0
        live = [s for s in range(a, b) if table.held[s] >= 0]
        assert k == 0 or len(live) > 1
        assert all(table.held[s] >= k and table.pages[s][:k // 16] == table.pages[live[0]][:k // 16] for s in live if k)
    assert sum(max(sum(table.held[s] >= 0 for s in range(a, b)) - 1, 0) * k // 16
               for a, b, k in zip(first, first[1:], p)) == most(table) > 0
