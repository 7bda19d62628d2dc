"""Waits of the prompt kernel: tiles of few blocks, whose last products are still on their way when
the rows are done with the last logits, beside ones that keep the memory system busy; and a model of
the barriers of its products."""
import pytest
import torch

from test_gpu_paged import attend_reference, check_attend, dev, make_cache, status, tables  # noqa: F401


class Barrier:
    """Completes phase after phase; a wait for parity p passes unless the phase that is open has it."""

    def __init__(self):
        self.done = 0

    def passes(self, parity):
        return self.done & 1 != parity


def products(done, blocks):
    """The barriers of a product and of all, after `done` of them."""
    o, end = Barrier(), Barrier()
    o.done, end.done = done, int(done == blocks)
    return o, end


@pytest.mark.parametrize("blocks", range(1, 12))
def test_the_waits_for_products(blocks):
    # at block j, products 0 .. j - 2 are done for certain and product j is not begun
    for j in range(1, blocks):
        for done in range(j - 1, j + 1):
            assert products(done, blocks)[0].passes((j - 1) & 1) == (done == j)
    # at the end any of the last two may be open
    for done in range(max(blocks - 2, 0), blocks + 1):
        assert products(done, blocks)[1].passes(0) == (done == blocks)
        if done == blocks - 2:                          # which one barrier for all does not tell
            one = Barrier()
            one.done = done
            assert one.passes((blocks - 1) & 1)


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_tiles_of_few_blocks(dev, d, out_dtype):  # noqa: F811
    """Tiles of 1 to 8 blocks in one call with long ones, many times: the same bits, and right."""
    H, G, page = 2, 4, 16
    held = [0, 40, 100, 170, 230, 300, 400, 3000, 2500, 2900]
    new = [40, 30, 28, 25, 40, 33, 70, 64, 200, 130]
    n = sum(-(-(p + k) // page) for p, k in zip(held, new))
    cache = make_cache(dev, n, H, d, page, seed=51)
    table, lens, starts = tables(held, new, page, n, dev, seed=52)
    q = (torch.randn((sum(new), H * G, d), generator=torch.Generator().manual_seed(53)) * 0.02).bfloat16().to(dev)
    first, lse = cache.attend(table, lens, q, starts=starts, max_new=200, out_dtype=out_dtype, want_lse=True)
    check_attend(first, lse, attend_reference(cache, table, held, new, q, page), out_dtype)
    flush = torch.empty(160 << 20, dtype=torch.uint8, device=dev)
    for i in range(40):
        if i % 2:
            flush.fill_(i)                              # the bytes come from HBM, late
        again, lse2 = cache.attend(table, lens, q, starts=starts, max_new=200, out_dtype=out_dtype, want_lse=True)
        assert torch.equal(again, first) and torch.equal(lse2, lse)
    assert status()[0] == 0
