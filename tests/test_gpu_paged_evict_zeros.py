"""Eviction of rows of zeros whose old scale lies far above that of their new block."""
import numpy as np
import pytest
import torch

from test_gpu_paged import dev, make_cache, tables  # noqa: F401
from test_gpu_paged_evict import run_and_check, to_table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [31, 32, 40, 100])
def test_zeros_under_a_scale_far_above(dev, d, top):  # noqa: F811
    """Zeros (of both signs) stay zeros where the old scale over the new one passes what fp32 holds, beside
    rows of the smallest scale, beside NaN, and in blocks of nothing else."""
    held, H, page, keep = [160], 2, 16, 48
    cache = make_cache(dev, 30, H, d, page, seed=2)
    table, lens, _ = tables(held, [0], page, 15, dev, seed=3)
    ids = table[0, :10].long().cpu()
    for pages, scale in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
        b = pages.view(torch.uint8)
        for j, pg in enumerate(ids.tolist()):
            scale[pg] = 2.0 ** (top if j % 2 else -96)
            if j % 2:
                b[pg, :, 3::2] = 0                      # (the other rows of these blocks have values)
                b[pg, :, 5, ::3] = 128                  # -0
                b[pg, :, 7, 1::5] = 127                 # NaN among zeros
    # kept: a block of rows of the smallest scale with zeros among them, one of zeros alone, one of all kinds
    m = torch.zeros((1, H, table.shape[1] * page))
    small = [p * 16 + r for p in (0, 2, 4) for r in (0, 1, 6)]
    zeros = [p * 16 + r for p in (1, 3, 5) for r in (3, 5, 7)]
    alone = [p * 16 + r for p in (7,) for r in (3, 5, 7, 9, 11, 13, 15)] + [9 * 16 + r for r in (3, 5, 7, 9, 11, 13, 15)]
    rest = [9 * 16 + 14] + [8 * 16 + r for r in range(14)]
    stay = sorted(set(small + zeros + alone + rest))
    m[..., stay] = 1.0
    keep = len(stay)
    to = to_table(table, 1, -(-keep // page), 30)
    run_and_check(dev, cache, table, lens, held, m, to, keep, 0, 0, page)
    out = [p.view(torch.uint8)[to[0, 0].long()] for p in (cache.k_pages, cache.v_pages)]
    first = np.array(stay[:16])
    for row in np.flatnonzero(np.isin(first, [p for p in zeros if p % 16 == 3])):
        assert all((o[:, row] == 0).all() for o in out)
