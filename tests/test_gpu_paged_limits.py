"""Paged attention at the ends of what an int holds: lengths whose tokens' positions pass it."""
import pytest
import torch

from test_gpu_paged import dev, make_cache, status  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 4, 40])
@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 31 - 1500, 10 ** 6])
def test_positions_past_the_table_see_what_it_holds(dev, length, new):  # noqa: F811
    """Recorded, and every token of the sequence sees the whole of its row of the table; the other
    sequence of the call is as without it."""
    d, H, G, page = 64, 2, 4, 16
    cache = make_cache(dev, 5, H, d, page, seed=71)
    table = torch.tensor([[3, 0], [1, 4]], dtype=torch.int32, device=dev)
    q = (torch.randn((new + 2, H * G, d), generator=torch.Generator().manual_seed(72)) * 0.02).bfloat16().to(dev)
    out, lse = cache.attend(table, torch.tensor([length, 20], dtype=torch.int32, device=dev), q, max_new=new,
                            starts=torch.tensor([0, new, new + 2], dtype=torch.int32, device=dev), want_lse=True)
    assert status()[0] == 6
    rows = torch.tensor([[3, 0]] * new + [[1, 4]] * 2, dtype=torch.int32, device=dev)
    held = torch.tensor([31] * new + [20, 21], dtype=torch.int32, device=dev)
    want, wl = cache.attend(rows, held, q, want_lse=True)
    assert status()[0] == 0
    assert torch.allclose(out, want, rtol=1e-5, atol=1e-4) and torch.allclose(lse, wl, rtol=1e-5, atol=1e-5)
