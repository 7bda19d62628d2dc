"""Attention weights for many query rows (tcgen05): tiles cut over the SMs and added up, rows that stay
for all tiles of a head, edges of tiles and blocks, batches with few and many rows."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import dev, hide_rest, make_cache, status, tables  # noqa: F401
from test_gpu_paged_weigh import check, keys_of, start_mass

pytestmark = pytest.mark.gpu


def logits(cache, table, held, new, q, page):
    """For each sequence and head: logits [n][G][T] and the sums of their magnitudes, in 64 bits."""
    H, G, d = cache.H, q.shape[1] // cache.H, cache.d
    out, at = {}, 0
    for s, (p, n) in enumerate(zip(held, new)):
        if p >= 0 and n > 0:
            for h in range(H):
                k = keys_of(cache, table, s, h, p + n, page)
                x = q[at:at + n, h * G:h * G + G].double().cpu().numpy()
                gone = np.arange(p + n) > p + np.arange(n)[:, None]
                out[s, h] = (np.where(gone[:, None], -math.inf, x @ k.T / math.sqrt(d)), np.abs(x) @ np.abs(k).T / math.sqrt(d))
        at += n
    return out


def normalisers(x, tokens, H, G, held, new):
    lse, at = torch.full((tokens, H * G), -math.inf), 0
    for s, (p, n) in enumerate(zip(held, new)):
        for h in range(H):
            if (s, h) in x:
                lse[at:at + n, h * G:h * G + G] = torch.logsumexp(torch.from_numpy(x[s, h][0]), -1).float()
        at += n
    return lse


def reference(x, lse, mass, H, G, held, new):
    """As the tests of few rows have it: 2^-21 of the magnitudes, of lse, 2^-20; 2^-24 for each addition."""
    out, tol, at = mass.double().numpy().copy(), np.zeros(mass.shape), 0
    for s, (p, n) in enumerate(zip(held, new)):
        for h in range(H):
            if (s, h) in x:
                l = lse[at:at + n, h * G:h * G + G].double().numpy()[..., None]
                w = np.where(l == -math.inf, 0.0, np.exp(np.where(l == -math.inf, -math.inf, x[s, h][0] - np.where(l == -math.inf, 0.0, l))))
                out[s, h, p:p + n] = 0.0
                out[s, h, :p + n] += w.sum((0, 1))
                err = 2.0 ** -21 * x[s, h][1] + 2.0 ** -21 * np.where(l == -math.inf, 0.0, np.abs(l)) + 2.0 ** -20
                tol[s, h, :p + n] = (w * err).sum((0, 1)) + (n * G + 32) * 2.0 ** -24 * np.abs(out[s, h, :p + n])
        at += n
    return out, tol


CASES = [
    # d, H, G, page, held, new
    (128, 1, 2, 64, [0], [2600]),                    # 41 blocks of rows, tiles cut over many SMs
    (64, 1, 4, 32, [0], [1700]),
    (128, 2, 4, 64, [3000], [300]),                  # more blocks than stay
    (64, 2, 3, 16, [5, 600, 0], [400, 333, 90]),
    (128, 3, 4, 128, [2050, 1000, 511], [37, 64, 9]),     # rows that stay: one, two blocks
    (64, 2, 4, 64, [1999, 256, 255, 257], [250, 33, 64, 10]),
    (128, 1, 40, 16, [300, 30], [1, 2]),             # many heads, few tokens
    (64, 1, 1, 16, [255, 256, 257, 0], [33, 128, 129, 256]),   # ends of tiles and blocks
    (128, 2, 7, 16, [100, 3, 50, 0], [5, 1, 4, 40]),      # few rows beside many
    (128, 1, 4, 1024, [1500], [260]),
    (64, 1, 130, 16, [700], [1]),                    # more rows than a block for one token
]


@pytest.mark.parametrize("case", CASES)
def test_many_rows(dev, case):
    d, H, G, page, held, new = case
    need = sum(-(-(p + n) // page) for p, n in zip(held, new))
    table, lens, starts = tables(held, new, page, need, dev, seed=3)
    cache = make_cache(dev, need, H, d, page, seed=2)
    hide_rest(cache, table, held, new, page)
    q = (torch.randn((sum(new), H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    x = logits(cache, table, held, new, q, page)
    lse = normalisers(x, sum(new), H, G, held, new)
    lse[sum(new) // 2] = -math.inf                     # a row that saw nothing
    mass = start_mass(table, H, page, held)
    want, tol = reference(x, lse, mass, H, G, held, new)
    kw = {} if max(new) == 1 else dict(starts=starts, max_new=max(new))
    got = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), **kw)
    check(got, want, tol)
    assert status()[0] == 0
    again = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), **kw)
    assert torch.equal(got.nan_to_num(nan=-1.0), again.nan_to_num(nan=-1.0))
    # the workspace is as it was: the attention that shares it runs as before
    cache.attend(table, lens, q, **kw)
    third = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), **kw)
    assert torch.equal(got.nan_to_num(nan=-1.0), third.nan_to_num(nan=-1.0))
    assert status()[0] == 0


def test_nan_keys_and_rows(dev):
    """NaN keys that rows see, whose normalisers are then NaN; behind rows that do not; rows that saw
    nothing beside a NaN; nobody's rows."""
    d, H, G, page, held, new = 64, 1, 2, 16, [500], [60]
    table, lens, starts = tables(held, new, page, 40, dev, seed=3)
    cache = make_cache(dev, 40, H, d, page, seed=2)
    hide_rest(cache, table, held, new, page)
    q = (torch.randn((70, G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    x = logits(cache, table, held, new, q[:60], page)
    lse = torch.full((70, G), math.nan)
    lse[:60] = normalisers(x, 60, H, G, held, new)
    cache.k_pages.view(torch.uint8)[int(table[0, 550 // 16]), 0, 550 % 16] = 127   # a key that tokens 50 .. see
    lse[50:60] = -math.inf                             # (say they were left out)
    mass = start_mass(table, H, page, held)
    want, tol = reference(x, lse[:60], mass, H, G, held, new)
    got = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), starts=starts)
    check(got, want, tol)
    lse[55] = math.nan
    got = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), starts=starts)
    assert torch.isnan(got[0, 0, :556]).all()
    check(got[0, 0, 556:560], want[0, 0, 556:560], tol[0, 0, 556:560] + 1e-30)
    assert status()[0] == 0


def test_bad_pages(dev):
    d, H, G, page, held, new = 128, 2, 4, 64, [900], [40]
    table, lens, starts = tables(held, new, page, 20, dev, seed=3, spare=0)
    cache = make_cache(dev, 20, H, d, page, seed=2)
    q = (torch.randn((40, H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    _, lse = cache.attend(table, lens, q, starts=starts, want_lse=True)
    mass = torch.ones((1, H, table.shape[1] * page), device=dev)
    good = cache.weigh(table, lens, q, lse, mass.clone(), starts=starts)
    for bad in (-1, 20, 2 ** 31 - 1):
        worse = table.clone()
        worse[0, 5] = bad
        got = cache.weigh(worse, lens, q, lse, mass.clone(), starts=starts)
        assert status()[0] == 6
        assert (got[..., 320:384] == 1).all() and torch.equal(got[..., :320], good[..., :320])
        assert torch.equal(got[..., 384:], good[..., 384:])
    for n in (table.shape[1] * page - 40, table.shape[1] * page - 39, 2 ** 31 - 1):
        cache.weigh(table, torch.tensor([n], dtype=torch.int32, device=dev), q, lse, mass.clone(), starts=starts)
        assert status()[0] == (0 if n == table.shape[1] * page - 40 else 6)
    again = cache.weigh(table, lens, q, lse, mass.clone(), starts=starts)
    assert torch.equal(again, good) and status()[0] == 0


def test_strided_queries_and_captured(dev):
    d, H, G, page, held, new = 128, 2, 4, 64, [700, 20], [80, 3]
    table, lens, starts = tables(held, new, page, 20, dev, seed=3)
    cache = make_cache(dev, 20, H, d, page, seed=2)
    hide_rest(cache, table, held, new, page)
    wide = (torch.randn((83, 2, H * G, 2 * d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    q = wide[:, 1, :, d:]
    _, lse = cache.attend(table, lens, q, starts=starts, want_lse=True)
    mass = torch.zeros((2, H, table.shape[1] * page), device=dev)
    want = cache.weigh(table, lens, q.contiguous(), lse, mass.clone(), starts=starts)
    got = mass.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.weigh(table, lens, q, lse, got, starts=starts)
    graph.replay()
    assert torch.equal(got, want)
    graph.replay()
    twice = cache.weigh(table, lens, q, lse, want.clone(), starts=starts)
    assert torch.equal(got, twice)
