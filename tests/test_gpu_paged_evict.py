"""Eviction by accumulated weight against its 64-bit oracle: which positions stay, what the new pages
hold bit for bit, ties, NaN, sizes over clusters of CTAs, bad pages, capture."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as op
from test_gpu_paged import dev, make_cache, same_codes, status, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def to_table(table, rows, pages, n_pages, seed=11):
    """Pages that `table` does not hold."""
    used = set(table.flatten().tolist())
    free = [p for p in range(n_pages) if p not in used]
    order = torch.randperm(len(free), generator=torch.Generator().manual_seed(seed)).tolist()
    return torch.tensor([free[i] for i in order[:rows * pages]], dtype=torch.int32).view(rows, pages)


def expect(cache, table, held, to, kept, page):
    out = []
    for pages, scale in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
        b, sc = pages.view(torch.uint8).cpu().numpy().copy(), scale.cpu().numpy().astype(np.float64).copy()
        old, old_sc = b.copy(), sc.copy()
        for s, p in enumerate(held):
            if p < 0:
                continue
            for h in range(b.shape[1]):
                at = kept[s][h]
                for j in range(0, len(at), 16):
                    src = [(int(table[s, t // page]), t % page) for t in at[j:j + 16]]
                    codes = np.stack([old[i, h, r] for i, r in src])
                    new, scale_ = op.store_block(codes, [old_sc[i, h, r // 16] for i, r in src])
                    pg = int(to[s, j // page])
                    b[pg, h, j % page:j % page + len(src)] = new
                    sc[pg, h, j % page // 16] = scale_
        out += [b, sc]
    return out


def run_and_check(dev, cache, table, lens, held, mass, to, keep, sinks, window, page, kept=None):
    n, H = len(held), cache.H
    kept = kept or [[op.kept(mass[s, h, :p].tolist(), keep, sinks, window) for h in range(H)] if p >= 0 else None
                    for s, p in enumerate(held)]
    want = expect(cache, table.cpu().numpy(), held, to.cpu().numpy(), kept, page)
    new_mass = torch.full((n, H, keep + 3), -5.0, device=dev)
    before = mass.clone().to(dev)
    lens_out, got = cache.evict(table, lens, before, to.to(dev), keep, sinks=sinks, window=window, new_mass=new_mass)
    assert torch.equal(before.nan_to_num(nan=-9.0).cpu(), mass.nan_to_num(nan=-9.0))
    assert lens_out.tolist() == [min(p, keep) for p in held]
    got, nm = got.cpu(), new_mass.cpu()
    for s, p in enumerate(held):
        for h in range(H):
            at = kept[s][h] if p >= 0 else []
            assert got[s, h].tolist() == at + [-1] * (keep - len(at)), (s, h)
            assert torch.equal(nm[s, h, :len(at)].nan_to_num(nan=-9.0), mass[s, h, at].nan_to_num(nan=-9.0))
            assert (nm[s, h, len(at):] == -5).all()
    same_codes(cache.k_pages, want[0])
    same_codes(cache.v_pages, want[2])
    assert np.array_equal(cache.k_scale.cpu().numpy().astype(np.float64), want[1])
    assert np.array_equal(cache.v_scale.cpu().numpy().astype(np.float64), want[3])
    assert status()[0] == 0


CASES = [
    # d, H, page, held, keep, sinks, window
    (128, 2, 16, [0, 1, 15, 16, 17, 40, 100, -1], 16, 0, 0),
    (128, 1, 64, [300], 100, 4, 32),
    (64, 3, 32, [77, 200, 33], 33, 1, 0),
    (64, 2, 16, [50, -1, 51, 49], 50, 3, 47),         # sinks and window are all that stays
    (128, 2, 64, [65, 64, 63], 64, 0, 0),             # one too many
    (64, 1, 128, [500, 9], 1, 0, 0),                  # the largest alone
    (64, 1, 16, [30], 1, 1, 0),
    (64, 1, 16, [30], 1, 0, 1),
    (128, 2, 1024, [700, 1500], 350, 2, 7),
]


@pytest.mark.parametrize("case", CASES)
def test_evict(dev, case):
    d, H, page, held, keep, sinks, window = case
    cache = make_cache(dev, 60, H, d, page, seed=2)
    table, lens, _ = tables(held, [0] * len(held), page, 30, dev, seed=3)
    g = torch.Generator().manual_seed(4)
    mass = torch.rand((len(held), H, table.shape[1] * page + 5), generator=g)
    to = to_table(table, len(held), -(-keep // page), 60)
    run_and_check(dev, cache, table, lens, held, mass, to, keep, sinks, window, page)


@pytest.mark.parametrize("kind", ["equal", "few levels", "zeros", "negative", "special", "nan"])
def test_ties_and_values_of_every_kind(dev, kind):
    held, H, page, d, keep = [200, 90], 2, 16, 64, 48
    cache = make_cache(dev, 60, H, d, page, seed=2)
    table, lens, _ = tables(held, [0, 0], page, 30, dev, seed=3)
    g = torch.Generator().manual_seed(4)
    shape = (2, H, table.shape[1] * page)
    mass = {"equal": torch.full(shape, 0.25), "few levels": torch.randint(0, 4, shape, generator=g).float(),
            "zeros": torch.where(torch.rand(shape, generator=g) < 0.5, 0.0, -0.0),
            "negative": -torch.rand(shape, generator=g), "nan": torch.full(shape, math.nan),
            "special": torch.tensor([math.inf, -math.inf, math.nan, 0.0, -0.0, 1e-45, -1e-45, 3e38, 1.0])[
                torch.randint(0, 9, shape, generator=g)]}[kind]
    to = to_table(table, 2, 3, 60)
    run_and_check(dev, cache, table, lens, held, mass, to, keep, 2, 5, page)


def fast_kept(m, keep, sinks, window):
    """op.kept of finite, distinct or tied weights, by a stable sort."""
    n = len(m)
    if n <= keep:
        return list(range(n))
    mid = np.arange(sinks, n - window)
    order = mid[np.argsort(-m[mid].astype(np.float64), kind="stable")][:keep - sinks - window]
    return sorted(list(range(sinks)) + order.tolist() + list(range(n - window, n)))


@pytest.mark.parametrize("levels", [0, 7])
@pytest.mark.parametrize("n,H,lengths,keep", [(1, 1, [70001], 3001), (2, 2, [40000, 9000], 20000), (1, 3, [8193], 4096),
                                              (40, 8, [900, 1300], 700), (3, 1, [100003, 5, 65536], 999)])
def test_long_rows_over_clusters(dev, n, H, lengths, keep, levels):
    held, page, d = [lengths[i % len(lengths)] for i in range(n)], 64, 64
    need = sum(-(-p // page) for p in held)
    to_pages = -(-keep // page)
    total = need + n * to_pages
    cache = make_cache(dev, total, H, d, page, seed=2)
    table, lens, _ = tables(held, [0] * n, page, need, dev, seed=3)
    g = torch.Generator().manual_seed(4)
    mass = torch.randn((n, H, table.shape[1] * page), generator=g).mul(3).exp()
    if levels:
        mass = torch.randint(0, levels, mass.shape, generator=g).float()
    kept = [[fast_kept(mass[s, h, :p].numpy(), keep, 4, 33) for h in range(H)] for s, p in enumerate(held)]
    to = to_table(table, n, to_pages, total)
    run_and_check(dev, cache, table, lens, held, mass, to, keep, 4, 33, page, kept=kept)


def test_scales_far_apart_and_special_codes(dev):
    """Rows whose scales lie up to 2^196 apart in one block, zeros, NaN bytes, a scale that goes down."""
    held, H, page, d, keep = [96], 1, 16, 64, 40
    cache = make_cache(dev, 12, H, d, page, seed=5)
    table, lens, _ = tables(held, [0], page, 6, dev, seed=3, spare=0)
    b = cache.k_pages.view(torch.uint8)
    b[int(table[0, 1]), 0, 2] = 127
    b[int(table[0, 2]), 0] = 0                                        # nothing but zeros
    b[int(table[0, 3]), 0] = 129                                      # the smallest magnitude, negative
    b[int(table[0, 4]), 0, :, 1:] = 255
    for i, e in enumerate((-96, 100, 0, 17, 3, -20)):
        cache.k_scale[int(table[0, i])] = 2.0 ** e
        cache.v_scale[int(table[0, i])] = 2.0 ** (-e if e < 90 else 90)
    g = torch.Generator().manual_seed(4)
    to = to_table(table, 1, 3, 12)
    for stay in ([0, 5], [2, 3], [3], [4], [0, 1, 2, 3, 4, 5]):       # pages that are heavy
        mass = torch.rand((1, 1, 96), generator=g)
        for i in stay:
            mass[0, 0, 16 * i:16 * i + 16] += 1
        run_and_check(dev, cache, table, lens, held, mass, to, keep, 0, 0, page)


def test_shared_pages_are_read_and_stay(dev):
    """Two sequences over the same pages: each gets its own copy, and the pages keep their bytes."""
    H, page, d, keep = 2, 16, 128, 32
    cache = make_cache(dev, 20, H, d, page, seed=5)
    table = torch.tensor([[3, 7, 1, 9], [3, 7, 1, 4]], dtype=torch.int32, device=dev)
    lens = torch.tensor([60, 55], dtype=torch.int32, device=dev)
    mass = torch.rand((2, H, 64), generator=torch.Generator().manual_seed(4))
    before = cache.k_pages.view(torch.uint8).clone()
    to = to_table(table.cpu(), 2, 2, 20)
    run_and_check(dev, cache, table, lens, [60, 55], mass, to, keep, 1, 4, page)
    old = [1, 3, 4, 7, 9]
    assert torch.equal(cache.k_pages.view(torch.uint8)[old], before[old])


def test_bad_entries(dev):
    H, page, d, keep = 1, 16, 64, 32
    held = [40, 50]
    cache = make_cache(dev, 20, H, d, page, seed=5)
    table, lens, _ = tables(held, [0, 0], page, 8, dev, spare=0)
    mass = torch.rand((2, H, table.shape[1] * page), generator=torch.Generator().manual_seed(4)).to(dev)
    to = to_table(table, 2, 2, 20).to(dev)

    def run(table, lens, to):
        c = make_cache(dev, 20, H, d, page, seed=5)
        n, kept = c.evict(table, lens, mass, to, keep)
        return status()[0], c.k_pages.view(torch.uint8), n.tolist(), kept

    st, good, n, kept = run(table, lens, to)
    assert st == 0 and n == [32, 32]
    for bad in (20, -1, 2 ** 31 - 1):
        worse = to.clone()
        worse[0, 1] = bad
        st, got, n, k = run(table, lens, worse)
        assert st == 6 and torch.equal(k, kept)
        same = [p for p in range(20) if p != int(to[0, 1])]
        assert torch.equal(got[same], good[same])
        assert torch.equal(got[int(to[0, 1])], make_cache(dev, 20, H, d, page, seed=5).k_pages.view(torch.uint8)[int(to[0, 1])])
        worse = table.clone()
        worse[1, 0] = bad
        st, got, n, k = run(worse, lens, to)
        assert st == 6 and torch.equal(k, kept) and torch.equal(got[to[0].long()], good[to[0].long()])
    st, got, n, k = run(table, torch.tensor([40, 2 ** 31 - 1], dtype=torch.int32, device=dev), to)
    assert st == 6 and n == [32, 32] and torch.equal(k[0], kept[0]) and int(k.max()) < table.shape[1] * page


def test_captured_and_replayed(dev):
    H, page, d, keep = 2, 16, 64, 48
    held = [60, 100]
    cache = make_cache(dev, 40, H, d, page, seed=5)
    table, lens, _ = tables(held, [0, 0], page, 20, dev)
    to = to_table(table, 2, 3, 40).to(dev)
    g = torch.Generator().manual_seed(4)
    mass = torch.rand((2, H, table.shape[1] * page), generator=g).to(dev)
    new_mass = torch.zeros((2, H, 48), device=dev)
    kept, new_lens = torch.zeros((2, H, keep), dtype=torch.int32, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    args = dict(sinks=1, window=3, kept=kept, new_mass=new_mass, new_lens=new_lens)
    cache.evict(table, lens, mass, to, keep, **args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.evict(table, lens, mass, to, keep, **args)
    mass.copy_(torch.rand(mass.shape, generator=g))
    lens.copy_(torch.tensor([55, 20], dtype=torch.int32))
    graph.replay()
    a = [t.clone() for t in (kept, new_lens, cache.k_pages.view(torch.uint8))]
    cache.evict(table, lens, mass, to, keep, **args)
    assert all(torch.equal(x, y) for x, y in zip(a, (kept, new_lens, cache.k_pages.view(torch.uint8))))
    assert new_lens.tolist() == [48, 20]
    for s, p in enumerate([55, 20]):
        for h in range(H):
            at = op.kept(mass[s, h, :p].tolist(), keep, 1, 3)
            assert kept[s, h].tolist() == at + [-1] * (keep - len(at))


def test_rows_that_shared_memory_does_not_hold(dev):
    """More keys than a CTA has room for are read again in each pass."""
    H, page, d, keep, L = 160, 1024, 64, 300, 50001
    need = -(-L // page)
    cache = make_cache(dev, need + 1, H, d, page, seed=5)
    table, lens, _ = tables([L], [0], page, need, dev, spare=0)
    mass = torch.randint(0, 5000, (1, H, need * page), generator=torch.Generator().manual_seed(4)).float()
    to = to_table(table.cpu(), 1, 1, need + 1).to(dev)
    n, kept = cache.evict(table, lens, mass.to(dev), to, keep, sinks=2, window=20)
    assert n.tolist() == [keep] and status()[0] == 0
    for h in range(H):
        assert kept[0, h].tolist() == fast_kept(mass[0, h, :L].numpy(), keep, 2, 20)
