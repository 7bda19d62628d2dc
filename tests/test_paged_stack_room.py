"""The example's stack: pages for what shedding moves, and shedding that is refused (no GPU)."""
import os
import sys

import pytest

from conftest import ROOT

sys.path.insert(0, os.path.join(ROOT, "examples"))


def stack(**kw):
    import paged_stack
    kw = {**dict(layers=1, batch=16, hidden=16, n_kv_heads=1, q_per_kv=1, head_dim=64, max_tokens=2000 + 64 + 2), **kw}
    return paged_stack.PagedStack(device="cpu", **kw)


def full(st, lengths):
    for s in range(len(lengths)):
        st.table.open(s)
    st.table.grow(lengths)
    st.table.advance(lengths)


@pytest.mark.parametrize("kw, keep", [({}, 2066), ({}, 1024), ({"keep": 1024}, 1024), ({"keep": 512}, 512), ({"keep": 1}, 1)])
@pytest.mark.parametrize("lengths", [[2000 - 37 * s for s in range(16)], [2066] * 16])
def test_a_nearly_full_pool_has_room_to_shed(lengths, kw, keep):
    """The example's sizes without shared prompts: twice, with the steps' tokens between."""
    st = stack(weights=True, **kw)
    full(st, lengths)
    for _ in range(2):
        to = st.table.shrink(keep)
        rows = [[p for p in r if p >= 0] for r in to.tolist()]
        assert [len(r) for r in rows] == [-(-min(h, keep) // 64) for h in st.table.held]
        new = {p for r in rows for p in r}
        assert not new & {p for r in st.table.pages for p in r} and max(new) < st.caches[0].k_pages.shape[0]
        st.table.shrunk()
        more = min(64, min(2066 - h for h in st.table.held))
        st.table.grow(more)
        st.table.advance(more)


def test_no_room_where_nothing_is_shed():
    assert stack().caches[0].k_pages.shape[0] == 16 * 33


@pytest.mark.parametrize("sinks, window", [(4, 64), (50, 1), (-1, 3), (3, -1)])
def test_shedding_that_is_refused_leaves_the_table_as_it_was(sinks, window):
    st = stack(weights=True, batch=2)
    full(st, [200, 100])
    before = list(st.table.free)
    with pytest.raises(ValueError):
        st.shed(50, sinks=sinks, window=window)
    assert st.table.free == before
    st.table.grow(1)                                   # nothing is pending
    st.table.advance(1)
