"""Captured steps of the paged example with idle places of the batch, and what comes after them: the
host's and the device's lengths stay the same, and pages are there for every token."""
import os
import sys

import pytest
import torch

from test_gpu_paged_stack import KW, hidden, mod, near, whole  # noqa: F401


@pytest.mark.parametrize("held", [[3, -1, 0], [-1, -1, 7]])
def test_lengths_of_idle_places_stay(held):
    from paper_2607_05061_gb300.paged import PageTable
    t = PageTable(3, 4, 12, page=16, device="cpu")
    for s, h in enumerate(held):
        if h >= 0:
            t.open(s)
    t.grow([max(h, 0) for h in held])
    t.advance([max(h, 0) for h in held])
    for i in range(1, 4):
        t.grow(1)
        t.advance_lens()
        t.advance_held(1)
        want = [h + i if h >= 0 else -1 for h in held]
        assert t.lens.tolist() == want and t.held == want


@pytest.mark.gpu
def test_replays_with_an_idle_place_and_what_follows(mod):  # noqa: F811
    lengths = [40, 0, 33, 62]
    xs = [hidden(n + 45, 60 + s) for s, n in enumerate(lengths)]
    want = whole(mod, xs)
    st = mod.PagedStack(**KW)
    for s in (0, 2, 3):
        st.table.open(s)
    st.chunk(torch.cat([xs[s][:lengths[s]] for s in (0, 2, 3)]), lengths)
    x_in = torch.zeros((4, KW["hidden"]), dtype=torch.bfloat16, device="cuda")
    y = st.capture(x_in)
    done = list(lengths)
    for _ in range(36):                                # over the ends of pages of 32
        x_in.copy_(torch.stack([x[d] for x, d in zip(xs, done)]))
        st.replay()
        for s in (0, 2, 3):
            assert near(y[s], want[s][done[s]])
            done[s] += 1
    st.check()
    assert st.table.lens.tolist() == st.table.held == [done[0], -1, done[2], done[3]]
    y = st.step(torch.stack([x[d] for x, d in zip(xs, done)]))
    assert all(near(y[s], want[s][done[s]]) for s in (0, 2, 3))
    done = [d + (s != 1) for s, d in enumerate(done)]
    st.table.open(1)                                   # the idle place is taken
    new = [8, 45, 1, 3]
    y = st.chunk(torch.cat([x[d:d + n] for x, d, n in zip(xs, done, new)]), new)
    st.check()
    for s, part in enumerate(torch.split(y, new)):
        assert near(part, want[s][done[s]:done[s] + new[s]])
    assert st.table.lens.tolist() == [d + n for d, n in zip(done, new)]
