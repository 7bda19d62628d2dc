"""Attention over shared prefixes whose groups' offsets go back: places that two groups claim."""
import pytest
import torch

from test_gpu_paged import attend_reference, dev, make_cache, status  # noqa: F401
from test_gpu_paged_shared import check, ints, shared_tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups, prefix", [([0, 5, 2, 6], [128, 0, 64]), ([0, 5, 2, 6], [64, 64, 192]),
                                            ([0, 6, 0, 6, 0, 3], [192, 64, 128, 64, 64])])
def test_places_of_two_groups(dev, groups, prefix):  # noqa: F811
    """All sequences share 192 positions, so any of the groups would do by itself: the first of those that
    overlap is taken, the others are recorded and left out, and every row sees each position once."""
    H, G, page, d, held = 2, 2, 16, 64, [200, 230, 210, 300, 192, 260]
    table, lens, _, total = shared_tables([0, 6], [192], held, [1] * 6, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    q = (torch.randn((6, H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    want = attend_reference(cache, table, held, [1] * 6, q, page)
    for _ in range(10):
        got, lse = cache.attend(table, lens, q, groups=ints(groups, dev), prefix=ints(prefix, dev), want_lse=True)
        assert status()[0] == 6
        check(got, lse, want, torch.float32)
