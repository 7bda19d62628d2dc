"""Precision of the paged attention's sums: values of one sign, for which every cut-off adds up, and
keys that leave all positions' weights alike, so that errors are relative to the result itself."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import dev, status  # noqa: F401
from test_gpu_paged_range import check, reference

gpu = pytest.mark.gpu

# Few rows: a block's products are formed from zero (two cut-offs below 2^-23), the weights have 22
# bits, blocks and warps add up rounded.
FEW = 2.0 ** -20
# Many rows: the products of 8 blocks of 64 add up cut off, 2 for each 16 positions: 64 times less than
# 2^-23 of what is there, which is half of the end on average.
MANY = 64 * 2.0 ** -23 / 2 + FEW


def cache_of(positions, H, d, page, seed):
    """Values in [1, 2), keys in (-1/8, 1/8), scales 1; pages in order."""
    from paper_2607_05061_gb300.paged import PagedCache
    g = torch.Generator().manual_seed(seed)
    n = -(-positions // page)
    shape = (n, H, page, d)
    k = torch.randint(0, 32, shape, generator=g, dtype=torch.uint8) + 128 * torch.randint(0, 2, shape, generator=g, dtype=torch.uint8)
    v = torch.randint(0x38, 0x40, shape, generator=g, dtype=torch.uint8)
    one = [torch.ones((n, H, page // 16), device="cuda") for _ in range(2)]
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(1, n)
    return PagedCache(*(t.cuda().view(torch.float8_e4m3fn) for t in (k, v)), *one), table


def worst(cache, q, out, lse, held, rows):
    """Largest relative error of the outputs, and largest error of the normalisers, of some rows."""
    H, d = cache.H, cache.d
    G = q.shape[1] // H
    err = off = 0.0
    for i in rows:
        for h in range(0, H * G, max(1, H * G - 1)):
            t = held + i + 1
            k, v = (x[:, h // G].double().reshape(-1, d)[:t] for x in (cache.k_pages, cache.v_pages))
            x = k @ q[i, h].double() / math.sqrt(d)
            y = torch.softmax(x, 0) @ v
            err = max(err, (out[i, h].double() / y - 1).abs().max().item())
            off = max(off, (lse[i, h].double() - torch.logsumexp(x, 0)).abs().item())
    return err, off


@gpu
@pytest.mark.parametrize("d,G,held,new", [(128, 4, 510, 1), (64, 4, 510, 1), (128, 4, 30000, 1), (128, 8, 2000, 3),
                                          (64, 3, 2000, 5)])
def test_few_rows(dev, d, G, held, new):  # noqa: F811
    cache, table = cache_of(held + new, 2, d, 64, 41)
    q = (torch.randn((new, 2 * G, d), generator=torch.Generator().manual_seed(42)) * 0.5).bfloat16().cuda()
    starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    out, lse = cache.attend(table, torch.tensor([held], dtype=torch.int32, device="cuda"), q, starts=starts,
                            max_new=new, want_lse=True)
    err, off = worst(cache, q, out, lse, held, range(new))
    assert err <= FEW and off <= FEW * 16 and status()[0] == 0


@gpu
@pytest.mark.parametrize("d,H,held,new", [(128, 8, 8192, 1856), (64, 8, 8192, 1856), (128, 8, 40000, 1856),
                                          (128, 1, 60000, 70), (64, 1, 0, 2000), (128, 2, 1000, 17)])
def test_many_rows(dev, d, H, held, new):  # noqa: F811
    """fp32 results of prompts that fill the SMs (tiles whole) and of a few tiles (cut in parts)."""
    G = 4
    cache, table = cache_of(held + new, H, d, 128, 43)
    q = (torch.randn((new, H * G, d), generator=torch.Generator().manual_seed(44)) * 0.5).bfloat16().cuda()
    starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    lens = torch.tensor([held], dtype=torch.int32, device="cuda")
    out, lse = cache.attend(table, lens, q, starts=starts, max_new=new, want_lse=True)
    err, off = worst(cache, q, out, lse, held, [0, new // 2 + 1, new - 1])
    assert err <= MANY and off <= FEW * 16
    again, lse2 = cache.attend(table, lens, q, starts=starts, max_new=new, want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2) and status()[0] == 0


@gpu
def test_bf16_results_of_very_long_contexts_keep_their_mean(dev):  # noqa: F811
    """Zero keys, values 1 or 2 with a probability of each column's own: columns' means spread over a
    bf16 binade, so that over 1024 columns the rounding leaves 2^-8 / sqrt(12 * 1024) = 3.5e-5 of the
    mean (four times that are allowed), and 256 blocks' products cut off 1024 times 2^-23 / 4 = 3.1e-5."""
    H, G, d, page, held, new = 8, 4, 128, 128, 262144, 1856
    cache, table = cache_of(page, H, d, page, 45)
    n = -(-(held + new) // page)
    from paper_2607_05061_gb300.paged import PagedCache
    g = torch.Generator(device="cuda").manual_seed(46)
    p = torch.rand((1, H, 1, d), generator=g, device="cuda") * 0.9 + 0.05
    v = torch.where(torch.rand((n, H, page, d), generator=g, device="cuda") < p, 0x40, 0x38).to(torch.uint8)
    one = [torch.ones((n, H, page // 16), device="cuda") for _ in range(2)]
    cache = PagedCache(torch.zeros_like(v).view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), *one)
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(1, n)
    q = torch.zeros((new, H * G, d), dtype=torch.bfloat16, device="cuda")
    out, _ = cache.attend(table, torch.tensor([held], dtype=torch.int32, device="cuda"), q, max_new=new,
                          starts=torch.tensor([0, new], dtype=torch.int32, device="cuda"), out_dtype=torch.bfloat16)
    i = new // 2
    t = held + i + 1
    y = 1 + sum((x.transpose(0, 1).reshape(H, -1, d)[:, :m] == 0x40).sum(1).double()
                for x, m in ((v[:t // page], t // page * page), (v[t // page:t // page + 1], t % page))) / t
    mean = (out[i].view(H, G, d)[:, 0].double() / y - 1).mean().item()
    assert abs(mean) <= 4 * 2.0 ** -8 / math.sqrt(12 * 1024) + 1024 * 2.0 ** -23 / 4


@gpu
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fall", [False, True])
def test_bases_that_move_between_chains(dev, fall, out_dtype):  # noqa: F811
    """Logits that rise (or fall) along 20000 keys: running sums are on other bases than what is added."""
    d, G, page, held, new = 128, 4, 64, 20000, 18
    cache, table = cache_of(held + new, 1, d, page, 47)
    cache.k_pages.view(torch.uint8).fill_(0x38)
    n = table.shape[1]
    for i in range(n):
        at = (n - 1 - i if fall else i) / n
        cache.k_scale[i] = 2.0 ** math.floor(8 * at - 5)
        cache.v_scale[i] = 2.0 ** (i % 7 - 3)
    q = torch.full((new, G, d), 0.6, device="cuda").bfloat16() * torch.tensor([1, -1, 0.3, 2.0], device="cuda").view(1, G, 1).bfloat16()
    out, lse = cache.attend(table, torch.tensor([held], dtype=torch.int32, device="cuda"), q, max_new=new,
                            starts=torch.tensor([0, new], dtype=torch.int32, device="cuda"), out_dtype=out_dtype, want_lse=True)
    check(out, lse, reference(cache, table, held, new, q, page))
    assert status()[0] == 0


def test_the_bounds_tell_one_f16_weight_from_two():
    """What the first bound is for: with weights of one f16 (11 bits) the same inputs miss it."""
    rng = np.random.default_rng(0)
    v = 1 + rng.integers(0, 8, (510, 128)) / 8
    x = rng.normal(size=510) * 0.5 * 0.3
    p = np.exp(x - x.max()) * 128
    one = p.astype(np.float16).astype(np.float64)
    two = one + (p - one).astype(np.float16).astype(np.float64)
    y = p @ v / p.sum()
    assert np.abs(one @ v / p.sum() / y - 1).max() > 4 * FEW
    assert np.abs(two @ v / p.sum() / y - 1).max() < FEW / 4
