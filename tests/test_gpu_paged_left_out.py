"""Single tokens that append leaves out for their positions: what a block's scale is behind them."""
import pytest
import torch

from test_gpu_paged import dev, make_cache, rotation, status, tables  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("stale", [2.0 ** 60, 2.0 ** 100, 2.0 ** -96])
def test_a_first_token_that_is_left_out(dev, d, dtype, stale):  # noqa: F811
    """A block's first token is left out, its second comes: as both in one call, whatever scale the page's
    earlier owner left; one that is not the first leaves the scale alone."""
    held, H, G, page = [16, 0, 33], 2, 3, 32
    table, lens, starts = tables(held, [2] * 3, page, 8, dev)
    n = len(held)
    cos, sin = (t.to(dev) for t in rotation(50, d // 2))
    x = torch.randn((2 * n, H * G + 2 * H, d), generator=torch.Generator().manual_seed(7)).to(dtype).to(dev)
    x[5] = x[4]                                        # (one scale for both, so that none is rounded twice)
    pos = torch.tensor([-1, 7, 50, 8, 9, 9], dtype=torch.int32, device=dev)       # (the first tokens of two of them)
    one, both = (make_cache(dev, 8, H, d, page) for _ in range(2))
    for cache in (one, both):
        cache.k_scale.fill_(stale)
        cache.v_scale.fill_(stale)
        for pages in (cache.k_pages, cache.v_pages):
            pages.view(torch.uint8).fill_(0)
    parts = lambda y: (y[:, :H * G], y[:, H * G:H * G + H], y[:, H * G + H:])  # noqa: E731
    both.append(table, lens, *parts(x), cos, sin, starts=starts, positions=pos)
    assert status()[0] == 6
    for i in range(2):
        before = one.k_scale.clone()
        one.append(table, lens + i, *parts(x[i::2].contiguous()), cos, sin, positions=pos[i::2].contiguous())
        assert status()[0] == (6 if i == 0 else 0)
        if i == 0:                                     # only the blocks that these tokens begin
            new = torch.zeros_like(before, dtype=torch.bool)
            for s in (0, 1):
                new[table[s, held[s] // page].long(), :, held[s] % page // 16] = True
            new[table[2, 1].long(), :, 0] = True       # (the third's token counts)
            assert torch.equal(one.k_scale[~new], before[~new])
    for a, b in ((one.k_scale, both.k_scale), (one.v_scale, both.v_scale), (one.k_pages, both.k_pages),
                 (one.v_pages, both.v_pages)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_later_token_that_is_left_out(dev):  # noqa: F811
    held, H, G, page, d = [17, 31], 2, 2, 16, 128
    table, lens, _ = tables(held, [1] * 2, page, 8, dev)
    cache = make_cache(dev, 8, H, d, page)
    before = [t.clone() for t in (cache.k_scale, cache.v_scale, cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8))]
    cos, sin = (t.to(dev) for t in rotation(50, d // 2))
    x = (torch.randn((2, H * G + 2 * H, d), generator=torch.Generator().manual_seed(7)) * 2.0 ** 20).to(dev)
    cache.append(table, lens, x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:], cos, sin,
                 positions=torch.tensor([50, -1], dtype=torch.int32, device=dev))
    assert status()[0] == 6
    after = (cache.k_scale, cache.v_scale, cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8))
    assert all(torch.equal(a, b) for a, b in zip(before, after))
