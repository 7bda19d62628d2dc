"""Outputs that a paged call makes itself, on a stream that is not the current one."""
import pytest
import torch

from test_gpu_paged import dev, make_cache, status, tables  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("handle", [False, True])
def test_outputs_are_not_memory_that_the_current_stream_still_uses(dev, handle):  # noqa: F811
    H, G, d, page, n = 2, 4, 128, 16, 64
    cache = make_cache(dev, 2 * n, H, d, page, seed=81)
    table, lens, _ = tables([9] * n, [1] * n, page, 2 * n, dev, seed=82)
    x = torch.randn((n, H * G + 2 * H, d), generator=torch.Generator().manual_seed(83)).bfloat16().to(dev)
    parts = x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]
    want_q = cache.append(table, lens, *parts)
    want, want_lse = cache.attend(table, lens, want_q, want_lse=True)
    side = torch.cuda.Stream()
    on = side.cuda_stream if handle else side
    torch.cuda.synchronize()
    # blocks of the outputs' sizes that the current stream will write late, and that are free for it
    used = [torch.empty_like(t) for t in (want_q, want, want_lse)]
    taken = {t.data_ptr() for t in used}
    torch.cuda._sleep(20_000_000)
    for t in used:
        t.fill_(7)
    del used, t
    q = cache.append(table, lens, *parts, stream=on)
    out, lse = cache.attend(table, lens, q, want_lse=True, stream=on)
    assert not taken & {t.data_ptr() for t in (q, out, lse)}
    torch.cuda.synchronize()
    assert torch.equal(q, want_q) and torch.equal(out, want) and torch.equal(lse, want_lse) and status()[0] == 0
