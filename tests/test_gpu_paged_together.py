"""Append at positions, shared prefixes, weights and eviction as they are used together: the example's
stack with sequences that share a prompt, decode, shed tokens and decode on."""
import numpy as np
import pytest
import torch

from oracle import paged as op
from test_gpu_paged import status
from test_gpu_paged_stack import hidden, mod, near  # noqa: F401

pytestmark = pytest.mark.gpu
KW = dict(layers=2, batch=6, hidden=256, n_kv_heads=2, q_per_kv=4, head_dim=64, max_tokens=400, page=16)


def shared_and_alone(mod, weights=True):
    """Two stacks in the same state: places 1 to 4 share 208 of place 0's 220 tokens, or hold copies."""
    prompt = hidden(220, 1)
    tails = [hidden(n, 20 + n) for n in (0, 30, 1, 17, 40)]
    st, alone = mod.PagedStack(weights=weights, **KW), mod.PagedStack(weights=weights, **KW)
    st.table.open(0)
    st.chunk(prompt, [220, 0, 0, 0, 0, 0])
    n = st.share(0, range(1, 5), 220)
    assert n == 208 and st.groups[1].tolist() == [208, 0]
    new = [0] + [len(prompt) - n + len(t) for t in tails[1:]] + [0]
    got = st.chunk(torch.cat([torch.cat([prompt[n:], t]) for t in tails[1:]]), new)
    for s in range(5):
        alone.table.open(s)
    whole = alone.chunk(torch.cat([torch.cat([prompt, t]) for t in tails]), [220 + len(t) for t in tails] + [0])
    want = torch.split(whole, [220 + len(t) for t in tails])
    assert near(got, torch.cat([w[n:] for w in want[1:]]))
    return st, alone


def test_shared_prompts_then_steps(mod):
    st, alone = shared_and_alone(mod)
    for i in range(3):
        x = hidden(6, 50 + i)
        a, b = st.step(x), alone.step(x)
        assert near(a[:5], b[:5])
    st.check()
    alone.check()
    # Weights: the same but for roundings at place 0 and at positions that a place read itself.  The shared
    # positions came with what place 0 had given them, its tokens 208 to 219 among it, which each place then
    # read once more: 12 tokens of 4 heads, one a row in all, give them at most 48 more.
    for m, n in zip(st.mass, alone.mass):
        for s in range(5):
            T, own = alone.table.held[s], 208 if s else 0
            assert torch.allclose(m[s, :, own:T], n[s, :, own:T], rtol=2 ** -4, atol=2 ** -4 * float(n[s, :, :T].mean()))
            more, slack = (m[s, :, :own] - n[s, :, :own]).sum(-1), 2 ** -4 * n[s, :, :own].sum(-1)
            assert (more >= -slack).all() and (more <= 48 * (own > 0) + slack).all()
    assert status()[0] == 0


def test_shedding_nothing_changes_nothing(mod):
    st, _ = shared_and_alone(mod)
    other, _ = shared_and_alone(mod)
    st.shed(300, sinks=2, window=8)                # more than any place holds: everything moves, nothing goes
    assert st.table.held == other.table.held and st.groups == (None, None)
    for i in range(2):
        x = hidden(6, 60 + i)
        assert near(st.step(x)[:5], other.step(x)[:5])
    st.check()


def test_shed_and_go_on(mod):
    """After an eviction: each head holds what the oracle keeps, steps append behind it at the tokens'
    own positions, and attention is over what the cache holds."""
    st, _ = shared_and_alone(mod)
    keep, H, d, page = 100, 2, 64, 16
    held, table = list(st.table.held), st.table.dev.cpu().clone()
    mass = [m.cpu().clone() for m in st.mass]
    before = [(c.k_pages.view(torch.uint8).cpu().numpy().copy(), c.k_scale.cpu().numpy().copy()) for c in st.caches]
    st.shed(keep, sinks=4, window=16)
    assert st.table.held == [100] * 5 + [-1] and st.table.seen == held and st.table.lens.tolist() == st.table.held

    def rows(pages, scale, table, s, h, at):
        ids = np.array([int(table[s, t // page]) for t in at])
        r = np.array(at) % page
        return op.E4M3[pages[ids, h, r]] * scale[ids, h, r // 16].astype(np.float64)[:, None]

    for i, c in enumerate(st.caches):
        now, ns = c.k_pages.view(torch.uint8).cpu().numpy(), c.k_scale.cpu().numpy()
        for s in (0, 3):
            for h in range(H):
                at = op.kept(mass[i][s, h, :held[s]].tolist(), keep, 4, 16)
                old = rows(*before[i], table, s, h, at)
                new = rows(now, ns, st.table.dev.cpu(), s, h, list(range(keep)))
                # a step of e4m3's smallest codes under the new scale, at most half of it off
                step = np.repeat(ns[[int(st.table.dev[s, t // page]) for t in range(0, keep, 16)], h, 0], 16)[:keep, None]
                assert (np.abs(new - old) <= step * 2.0 ** -10).all()
                assert torch.equal(st.mass[i][s, h, :keep].cpu(), mass[i][s, h, at])
    # a step: the first layer's attention against 64 bits over the cache as it is then
    x = hidden(6, 70)
    c, W = st.caches[0], st.layers[0]
    st.table.grow(1)
    qkv = torch.matmul(x, W["Wqkv"]).view(6, -1, d)
    q = c.append(st.table.dev, st.table.lens, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], st.cos, st.sin, positions=st.table.pos)
    o, lse = c.attend(st.table.dev, st.table.lens, q, want_lse=True)
    for s in (0, 3):
        turn = op.rotate(qkv[s, 5].float().cpu().numpy(), st.cos[held[s]].cpu().numpy(), st.sin[held[s]].cpu().numpy())
        assert np.abs(q[s, 5].float().cpu().numpy() - turn).max() <= 2.0 ** -8 * np.abs(turn).max()
        for hq in (0, 6):
            k, v = (rows(p.view(torch.uint8).cpu().numpy(), sc.cpu().numpy(), st.table.dev.cpu(), s, hq // 4, list(range(keep + 1)))
                    for p, sc in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)))
            y, l = op.attend(q[s, hq].double().cpu().numpy(), k, v)
            assert np.abs(o[s, hq].double().cpu().numpy() - y).max() <= 2.0 ** -15 * np.abs(v).max()
            assert abs(lse[s, hq].item() - l) <= 2.0 ** -15 * max(1.0, abs(l))
    assert status()[0] == 0


def test_captured_steps_after_shedding(mod):
    st, _ = shared_and_alone(mod)
    other, _ = shared_and_alone(mod)
    for t in (st, other):
        t.shed(120, sinks=4, window=16)
        t.table.grow(5)
    x = hidden(6, 80)
    y = st.capture(x)
    for i in range(3):
        x.copy_(hidden(6, 81 + i))
        st.replay()
        want = other.step(x)
        assert torch.equal(y[:5], want[:5])
    st.check()
    assert st.table.lens.tolist() == other.table.lens.tolist() and st.table.pos.tolist() == other.table.pos.tolist()
    assert st.table.seen == other.table.seen and all(torch.equal(a, b) for a, b in zip(st.mass, other.mass))


def test_more_tokens_in_a_chunk_after_shedding(mod):
    st, _ = shared_and_alone(mod)
    st.shed(64, sinks=0, window=64)                # the last 64 alone
    y = st.chunk(hidden(40, 90), [3, 20, 1, 16, 0, 0])
    assert torch.isfinite(y).all()
    assert st.table.held == [67, 84, 65, 80, 64, -1]
    st.check()
    assert status()[0] == 0
