"""Which rows of a call's tokens are whose, with idle places in the batch."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture()
def stack(monkeypatch):
    """The example's stack on the CPU, whose layers give back what they get."""
    import paged_stack
    from paper_2607_05061_gb300.paged import PageTable
    st = object.__new__(paged_stack.PagedStack)
    st.table = PageTable(4, 4, 16, page=16, device="cpu")
    st.calls = []

    def forward(x, starts=None, max_new=None):
        st.calls.append((starts.tolist(), max_new))
        return x
    st.forward = forward
    for s in (0, 2, 3):
        st.table.open(s)
    return st


def test_rows_of_an_idle_place_are_refused(stack):
    with pytest.raises(ValueError):
        stack.chunk(torch.zeros(3 + 20 + 5 + 1, 8), [3, 20, 5, 1])
    assert not stack.calls and stack.table.held == [0, -1, 0, 0] and not any(stack.table.pages)
    stack.chunk(torch.zeros(9, 8), [3, 20, 5, 1])
    assert stack.calls == [([0, 3, 3, 8, 9], 5)] and stack.table.lens.tolist() == [3, -1, 5, 1]


def test_too_few_and_too_many_rows_are_refused(stack):
    for n in (8, 10):
        with pytest.raises(ValueError):
            stack.chunk(torch.zeros(n, 8), [3, 0, 5, 1])
    stack.chunk(torch.zeros(9, 8), [3, 0, 5, 1])


def test_counts(stack):
    t = stack.table
    assert t.counts(2) == [2, 0, 2, 2] and t.counts([1, 7, 0, 3]) == [1, 0, 0, 3]
    assert t.starts([1, 7, 0, 3]).tolist() == [0, 1, 1, 1, 4]
    for bad in ([1, 2, 3], [1, 2, 3, -1]):
        with pytest.raises(ValueError):
            t.counts(bad)
