"""The paged layers together, as the example runs them: prompts in chunks of any size, single
tokens among them, and captured decode steps, against one pass over each whole sequence."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

KW = dict(layers=3, batch=4, hidden=256, n_kv_heads=2, q_per_kv=4, head_dim=64, max_tokens=240, page=32)


def hidden(n, seed):
    return torch.randn((n, KW["hidden"]), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


@pytest.fixture(scope="module")
def mod(cuda_device):
    import paged_stack
    return paged_stack


def whole(mod, xs):
    """Every sequence in one chunk."""
    st = mod.PagedStack(**KW)
    for s in range(4):
        st.table.open(s)
    y = st.chunk(torch.cat(xs), [len(x) for x in xs])
    st.check()
    return torch.split(y, [len(x) for x in xs])


def near(a, b):
    """Three layers of bf16 storage points; a chunk's end inside a block moves codes below 2^-6 of
    the block's scale by one step (2^-9 of it) at most."""
    d = (a.float() - b.float()).abs()
    return bool((d <= 2.0 ** -5 * (1 + b.float().abs())).all())


def test_chunks_and_single_tokens_equal_one_pass(mod):
    lengths = [130, 77, 200, 1]
    xs = [hidden(n, 10 + s) for s, n in enumerate(lengths)]
    want = whole(mod, xs)
    st = mod.PagedStack(**KW)
    for s in range(4):
        st.table.open(s)
    done, got = [0] * 4, [[] for _ in range(4)]
    plan = [[50, 1, 17, 1], [1, 60, 1, 0], [79, 1, 100, 0], [0, 15, 82, 0]]
    for new in plan:
        y = st.chunk(torch.cat([x[d:d + n] for x, d, n in zip(xs, done, new)]), new)
        for s, part in enumerate(torch.split(y, new)):
            got[s].append(part)
            done[s] += new[s]
    st.check()
    assert done == lengths and st.table.lens.tolist() == lengths
    assert all(near(torch.cat(g), w) for g, w in zip(got, want))


def test_captured_steps_equal_one_pass(mod):
    lengths = [40, 90, 33, 64]
    xs = [hidden(n + 6, 20 + s) for s, n in enumerate(lengths)]
    want = whole(mod, xs)
    st = mod.PagedStack(**KW)
    for s in range(4):
        st.table.open(s)
    st.chunk(torch.cat([x[:n] for x, n in zip(xs, lengths)]), lengths)
    y = st.step(torch.stack([x[n] for x, n in zip(xs, lengths)]))
    assert all(near(y[s], want[s][n]) for s, n in enumerate(lengths))
    st.table.grow(5)
    x_in = torch.zeros((4, KW["hidden"]), dtype=torch.bfloat16, device="cuda")
    y = st.capture(x_in)
    for j in range(1, 6):
        x_in.copy_(torch.stack([x[n + j] for x, n in zip(xs, lengths)]))
        st.graph.replay()
        assert all(near(y[s], want[s][n + j]) for s, n in enumerate(lengths))
    st.check()


def test_a_place_is_reused(mod):
    """A sequence that takes a closed one's pages sees nothing of it."""
    xs = [hidden(50, 30 + s) for s in range(4)]
    want = whole(mod, xs)
    st = mod.PagedStack(**KW)
    for s in (0, 1, 3):
        st.table.open(s)
    st.chunk(torch.cat([hidden(100, 40), hidden(30, 41), xs[3][:20]]), [100, 30, 0, 20])
    st.table.close(0)
    st.table.close(1)
    for s in (2, 0, 1):
        st.table.open(s)
    y = st.chunk(torch.cat([xs[0], xs[1], xs[2], xs[3][20:]]), [50, 50, 50, 30])
    st.check()
    got = torch.split(y, [50, 50, 50, 30])
    assert all(near(got[s], want[s]) for s in range(3)) and near(got[3], want[3][20:])
