"""Attention over the paged 8-bit cache where the scales of the values lie as far apart as the
format allows: no position's weight may get lost, whatever its values are.

Bounds: the fp32 sums of the logits (2^-21 of the sum of magnitudes), 2^-20 for exponentials and
sums, the weights' 22 or 11 bits, each of the row's weighted values; and the result's rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as op
from test_gpu_paged import dev, make_cache, status, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def reference(cache, table, held, new, q, page):
    """(y, lse, bound of the logits' errors, weighted largest |v|) of one sequence, in 64 bits."""
    H, d = cache.H, cache.d
    G = q.shape[1] // H
    ids = table.cpu().numpy()[0, :-(-(held + new) // page)]
    K, V = (op.E4M3[t.view(torch.uint8).cpu().numpy()[ids]] *
            np.repeat(s.cpu().numpy().astype(np.float64)[ids], 16, -1)[..., None]
            for t, s in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)))
    qd = q.double().cpu().numpy()
    y, lse, a, top = np.zeros(qd.shape), *(np.zeros(qd.shape[:2]) for _ in range(3))
    for i in range(new):
        for r in range(H * G):
            k, v = (x[:, r // G].reshape(-1, d)[:held + i + 1] for x in (K, V))
            y[i, r], lse[i, r] = op.attend(qd[i, r], k, v)
            w = np.exp(k @ qd[i, r] / math.sqrt(d) - lse[i, r])
            a[i, r] = (np.abs(k) @ np.abs(qd[i, r])).max() / math.sqrt(d)
            top[i, r] = w @ np.abs(v).max(1)
    return y, lse, a, top


def check(out, lse, want):
    y, wl, a, top = want
    eps = 2.0 ** -21 * a + 2.0 ** -20
    f32 = out.dtype == torch.float32
    tol = (2 * (eps + (2.0 ** -21 if f32 else 2.0 ** -11)) * top)[..., None] + (2.0 ** -23 if f32 else 2.0 ** -8) * np.abs(y)
    assert (np.abs(out.double().cpu().numpy() - y) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - wl) <= 2 * eps + 2.0 ** -20 * (1 + np.abs(wl))).all()


ORDERS = {"small first": lambda n: [0] * (n // 2) + [1] * (n - n // 2),
          "large first": lambda n: [1] * (n // 2) + [0] * (n - n // 2),
          "one large block": lambda n: [int(i == n // 3) for i in range(n)],
          "one small block": lambda n: [int(i != n // 3) for i in range(n)],
          "in turn": lambda n: [i & 1 for i in range(n)]}


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lo,hi", [(-96, 31), (-96, 100), (-45, 60)])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("d,H,held,new", [(64, 1, 300, 1), (128, 1, 2000, 1), (128, 2, 350, 5), (64, 1, 300, 40),
                                          (128, 1, 1900, 70)])
def test_equal_logits(dev, d, H, held, new, order, lo, hi, out_dtype):  # noqa: F811
    """Zero keys: every position has the same weight."""
    page, G = 16, 4
    n = -(-(held + new) // page)
    cache = make_cache(dev, n, H, d, page, seed=31)
    cache.k_pages.view(torch.uint8).zero_()
    table, lens, starts = tables([held], [new], page, n, dev, seed=32)
    for i, big in enumerate(ORDERS[order](n)):
        cache.v_scale[int(table[0, i])] = 2.0 ** (hi if big else lo)
    q = torch.randn((new, H * G, d), generator=torch.Generator().manual_seed(33)).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, starts=starts, max_new=new, out_dtype=out_dtype, want_lse=True)
    check(out, lse, reference(cache, table, held, new, q, page))
    assert status()[0] == 0


@pytest.mark.parametrize("new", [1, 40])
def test_zero_values_beside_large_ones(dev, new):  # noqa: F811
    """As `append` writes them: 16 tokens of zeros, then tokens of 1e15, equal logits."""
    d, H, G, page, held = 128, 1, 4, 64, 32
    cache = make_cache(dev, 4, H, d, page, seed=34)
    table, lens, starts = tables([0], [held + new], page, 4, dev)
    v = torch.full((held + new, H, d), 1e15, device=dev)
    v[:16] = 0
    cache.append(table, lens, None, torch.zeros_like(v), v, starts=starts)
    q = torch.randn((new, H * G, d), generator=torch.Generator().manual_seed(35)).bfloat16().to(dev)
    at = torch.tensor([0, new], dtype=torch.int32, device=dev)
    out, lse = cache.attend(table, lens + held, q, starts=at, max_new=new, want_lse=True)
    seen = torch.arange(held + 1, held + new + 1, device=dev).double()[:, None]
    kept = op.E4M3[op.round_e4m3(1e15 / 2.0 ** op.exponent(1e15))] * 2.0 ** op.exponent(1e15)
    assert ((out.double() / (kept * (seen - 16) / seen)[..., None] - 1).abs() <= 2.0 ** -18).all()
    assert ((lse.double() - torch.log(seen)).abs() <= 2.0 ** -18).all()


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("big", [True, False])
@pytest.mark.parametrize("held,new", [(300, 1), (2000, 1), (300, 40), (1900, 70)])
def test_weights_against_scales(dev, held, new, big, out_dtype):  # noqa: F811
    """Positions whose weights are as small as their values are large, first and last in their turn:
    both sorts count, though the weights of one are 2^-100 of the others'."""
    d, H, G, page = 128, 1, 4, 16
    n = -(-(held + new) // page)
    cache = make_cache(dev, n, H, d, page, seed=36)
    cache.k_pages.view(torch.uint8).fill_(0x38)                       # ones
    table, lens, starts = tables([held], [new], page, n, dev, seed=37)
    for i in range(n):
        large = (i < n // 2) == big
        cache.v_scale[int(table[0, i])] = 2.0 ** (60 if large else -40)
        cache.k_scale[int(table[0, i])] = 0.125 if large else 0.5
    # (0.5 - 0.125) sqrt(d) q = 100 log 2
    q = torch.full((new, H * G, d), 100 * math.log(2) / (0.375 * math.sqrt(d)), device=dev).bfloat16()
    out, lse = cache.attend(table, lens, q, starts=starts, max_new=new, out_dtype=out_dtype, want_lse=True)
    check(out, lse, reference(cache, table, held, new, q, page))
