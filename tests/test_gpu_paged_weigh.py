"""Attention weights of a cache's positions against 64 bits: rows, lengths, masks, NaN, strides, bad
tables, capture and streams."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as op
from test_gpu_paged import ATTEND, dev, hide_rest, make_cache, status, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def keys_of(cache, table, s, h, T, page):
    ids = table.cpu().numpy()[s, :-(-T // page)]
    k = op.E4M3[cache.k_pages.view(torch.uint8).cpu().numpy()[ids, h]]
    return (k * np.repeat(cache.k_scale.cpu().numpy().astype(np.float64)[ids, h], 16, -1)[..., None]).reshape(-1, cache.d)[:T]


def normalisers(cache, table, held, new, q, page):
    """fp32 normalisers [tokens][heads], from 64 bits."""
    H, G = cache.H, q.shape[1] // cache.H
    lse, at = np.full(q.shape[:2], -math.inf), 0
    for s, (p, n) in enumerate(zip(held, new)):
        if p >= 0:
            for h in range(H):
                k = keys_of(cache, table, s, h, p + n, page)
                x = q[at:at + n, h * G:h * G + G].double().cpu().numpy() @ k.T / math.sqrt(cache.d)
                for i in range(n):
                    lse[at + i, h * G:h * G + G] = torch.logsumexp(torch.from_numpy(x[i, :, :p + i + 1]), -1).numpy()
        at += n
    return torch.from_numpy(lse).float()


def reference(cache, table, held, new, q, lse, mass, page):
    """(mass, tolerance) in 64 bits."""
    H, G, d = cache.H, q.shape[1] // cache.H, cache.d
    out, tol, at = mass.double().numpy().copy(), np.zeros(mass.shape), 0
    qd, ld = q.double().cpu().numpy(), lse.double().numpy()
    for s, (p, n) in enumerate(zip(held, new)):
        if p >= 0 and n > 0:
            for h in range(H):
                k = keys_of(cache, table, s, h, p + n, page)
                out[s, h, p:p + n] = 0.0
                rows = 0
                for i in range(n):
                    for g in range(G):
                        r = (at + i, h * G + g)
                        if ld[r] == -math.inf:
                            continue
                        w = op.weights(qd[r], k[:p + i + 1], ld[r])
                        a = np.abs(k[:p + i + 1]) @ np.abs(qd[r]) / math.sqrt(d)
                        # fp32 sums of the logit; the normaliser's product and the exponent; the exponential
                        tol[s, h, :p + i + 1] += w * (2.0 ** -21 * a + 2.0 ** -21 * abs(ld[r]) + 2.0 ** -20)
                        out[s, h, :p + i + 1] += w
                        rows += 1
                # fp32 sums: each addition rounds by 2^-24 of what is there
                tol[s, h, :p + n] += (rows + 32) * 2.0 ** -24 * np.abs(out[s, h, :p + n])
        at += n
    return out, tol


def check(got, want, tol):
    got = got.double().cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    d = np.abs(got - want)[~nan]
    assert (d <= tol[~nan]).all(), (d / np.maximum(tol[~nan], 1e-300)).max()


def start_mass(table, H, page, held, extra=3, seed=9):
    """Sums so far; NaN where the new tokens and nobody's positions lie."""
    m = torch.rand((table.shape[0], H, table.shape[1] * page + extra), generator=torch.Generator().manual_seed(seed))
    for s, p in enumerate(held):
        m[s, :, max(p, 0):] = math.nan
    return m


@pytest.mark.parametrize("case", ATTEND)
def test_weigh(dev, case):
    d, H, G, page, held, new = case
    counts = new or [1] * len(held)
    cache = make_cache(dev, 40, H, d, page, seed=2)
    table, lens, starts = tables(held, counts, page, 40, dev, seed=3)
    hide_rest(cache, table, held, counts, page)
    q = (torch.randn((sum(counts), H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    lse = normalisers(cache, table, held, counts, q, page)
    mass = start_mass(table, H, page, held)
    want, tol = reference(cache, table, held, counts, q, lse, mass, page)
    got = [cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), starts=None if new is None else starts, max_new=m)
           for m in (max(counts), None, 1)]
    for x in got:
        check(x, want, tol)
    assert status()[0] == 0
    again = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), starts=None if new is None else starts,
                        max_new=max(counts))
    assert torch.equal(again.nan_to_num(nan=-1.0), got[0].nan_to_num(nan=-1.0))


def test_weights_sum_to_the_rows(dev):
    """With normalisers that attend returned, each row gives one in all."""
    held, H, G, page, d = [900, 0, 33, 2047], 2, 4, 32, 128
    counts = [3, 5, 1, 2]
    cache = make_cache(dev, 120, H, d, page, seed=2)
    table, lens, starts = tables(held, counts, page, 120, dev)
    hide_rest(cache, table, held, counts, page)
    q = (torch.randn((sum(counts), H * G, d), generator=torch.Generator().manual_seed(6)) * 0.02).bfloat16().to(dev)
    _, lse = cache.attend(table, lens, q, starts=starts, want_lse=True)
    mass = torch.zeros((4, H, table.shape[1] * page), device=dev)
    cache.weigh(table, lens, q, lse, mass, starts=starts)
    # a weight is off by 2^-20 and what lse is off by, and 2^-22 of the sum adds up per addition
    for s, n in enumerate(counts):
        assert (mass[s].double().sum(-1) - n * G).abs().max().item() <= n * G * 1e-4
    assert status()[0] == 0


def test_idle_places_rows_that_saw_nothing_and_nobodys_rows(dev):
    held, H, G, page, d = [20, -1, 5], 2, 2, 16, 64
    counts = [3, 2, 4]
    cache = make_cache(dev, 12, H, d, page, seed=3)
    table, lens, starts = tables(held, counts, page, 12, dev)
    hide_rest(cache, table, held, counts, page)
    q = (torch.randn((sum(counts) + 5, H * G, d), generator=torch.Generator().manual_seed(7)) * 0.02).bfloat16()
    q[9:] = math.nan                                    # rows past the last sequence
    q[3:5] = math.nan                                   # an idle place's
    q = q.to(dev)
    lse = torch.full((14, H * G), math.nan)
    lse[:9] = normalisers(cache, table, held, counts, q[:9], page)
    lse[1, 2] = -math.inf                               # saw nothing: gives nothing, whatever its product is
    cache.k_pages.view(torch.uint8)[int(table[0, 0]), 1, 3] = 127     # NaN keys of head 1, which all its rows see
    lse[0, 2:] = lse[2, 2:] = lse[1, 3] = -math.inf
    mass = start_mass(table, H, page, held)
    mass[1] = 5.0
    got = cache.weigh(table, lens, q, lse.to(dev), mass.to(dev), starts=starts).cpu()
    clean = lse[:9].clone()
    want, tol = reference(cache, table, held, counts, q[:9], clean, mass, page)
    check(got, want, tol)
    assert (got[1] == 5).all() and torch.isfinite(got[0, :, :23]).all() and torch.isnan(got[0, :, 23:]).all()
    assert status()[0] == 0


def test_nan_reaches_what_its_rows_see(dev):
    held, H, G, page, d = [30], 1, 2, 16, 128
    cache = make_cache(dev, 4, H, d, page, seed=3)
    table, lens, starts = tables(held, [4], page, 4, dev)
    q = (torch.randn((4, G, d), generator=torch.Generator().manual_seed(7)) * 0.02).bfloat16().to(dev)
    lse = normalisers(cache, table, held, [4], q, page)
    # a NaN key among the new tokens: the rows before it do not see it
    cache.k_pages.view(torch.uint8)[int(table[0, 2]), 0, 0] = 127     # position 32, the third new token
    got = cache.weigh(table, lens, q[:2], lse[:2].to(dev), torch.zeros((1, 1, table.shape[1] * page), device=dev),
                      starts=torch.tensor([0, 2], dtype=torch.int32, device=dev))
    assert torch.isfinite(got).all() and (got[0, 0, 32:] == 0).all()
    lse[3] = math.nan
    got = cache.weigh(table, lens, q, lse.to(dev), torch.zeros((1, 1, table.shape[1] * page), device=dev), starts=starts)
    assert torch.isnan(got[0, 0, :34]).all() and (got[0, 0, 34:] == 0).all()


def test_strides_and_long_contexts(dev):
    """Queries as columns of wider rows; contexts cut over all SMs."""
    held, H, G, page, d = [9001, 40, 3333], 2, 3, 64, 64
    cache = make_cache(dev, 210, H, d, page, seed=6)
    table, lens, _ = tables(held, [1] * 3, page, 210, dev, seed=7)
    wide = (torch.randn((3, 2, H * G, 2 * d), generator=torch.Generator().manual_seed(8)) * 0.02).bfloat16().to(dev)
    q = wide[:, 1, :, d:]
    lse = normalisers(cache, table, held, [1] * 3, q, page)
    mass = start_mass(table, H, page, held)
    want, tol = reference(cache, table, held, [1] * 3, q, lse, mass, page)
    check(cache.weigh(table, lens, q, lse.to(dev), mass.to(dev)), want, tol)


def test_bad_pages_and_tables(dev):
    held, H, G, page, d = [40, 20], 1, 2, 16, 64
    cache = make_cache(dev, 6, H, d, page, seed=3)
    table, lens, _ = tables(held, [1, 1], page, 6, dev, spare=0)
    q = (torch.randn((2, G, d), generator=torch.Generator().manual_seed(7)) * 0.02).bfloat16().to(dev)
    lse = normalisers(cache, table, held, [1, 1], q, page)
    mass = torch.ones((2, 1, 48), device=dev)
    good = cache.weigh(table, lens, q, lse.to(dev), mass.clone())
    bad = table.clone()
    bad[0, 1] = 6
    got = cache.weigh(bad, lens, q, lse.to(dev), mass.clone())
    assert status()[0] == 6
    assert torch.equal(got[0, :, :16], good[0, :, :16]) and torch.equal(got[0, :, 32:], good[0, :, 32:])
    assert (got[0, :, 16:32] == 1).all() and torch.equal(got[1], good[1])
    for length in (47, 48, 2 ** 31 - 1):                             # past the table's row
        cache.weigh(table, torch.tensor([length, 20], dtype=torch.int32, device=dev), q, lse.to(dev), mass.clone())
        assert status()[0] == (0 if length == 47 else 6)
    starts = torch.tensor([0, 9, 1], dtype=torch.int32, device=dev)
    cache.weigh(table, lens, q, lse.to(dev), mass.clone(), starts=starts)
    assert status()[0] == 6


def test_capture_and_streams(dev):
    held, H, G, page, d = [300, 77], 2, 4, 16, 128
    cache = make_cache(dev, 30, H, d, page, seed=4)
    table, lens, _ = tables(held, [1, 1], page, 30, dev, spare=2)
    q = (torch.randn((2, H * G, d), generator=torch.Generator().manual_seed(7)) * 0.02).bfloat16().to(dev)
    _, lse = cache.attend(table, lens, q, want_lse=True)
    mass = torch.zeros((2, H, table.shape[1] * page), device=dev)
    want = cache.weigh(table, lens, q, lse, mass.clone())
    twice = cache.weigh(table, lens, q, lse, want.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mass.clone()
    cache.weigh(table, lens, q, lse, got, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    got.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.weigh(table, lens, q, lse, got)
    assert (got == 0).all()
    graph.replay()
    assert torch.equal(got, want)
    graph.replay()
    assert torch.equal(got, twice)
