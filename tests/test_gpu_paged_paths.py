"""Paths of the paged kernels that the other tests do not reach: special values among several tokens,
outputs on 16-byte boundaries, large pages, pools past 4 GB under tcgen05, mixed batches in a graph,
idle places among offsets, parts in groups of 16, batches of very many sequences."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import (attend_reference, check_attend, dev, expect_append, fp32_rotate, hide_rest,  # noqa: F401
                            make_cache, rotation, same_codes, status, tables)

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def query(n, heads, d, seed, size=0.02):
    return (torch.randn((n, heads, d), generator=torch.Generator().manual_seed(seed)) * size).to(BF)


@pytest.mark.parametrize("rot", [0, 32])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_special_values_among_several_tokens(dev, d, dtype, rot):  # noqa: F811
    """Infinities, NaN and 2^108 in some tokens of a block, in the first and the last of them, blocks of
    nothing else, zeros and subnormals; blocks that go on with larger values."""
    H, page, held, new = 2, 32, [0, 5, 13], [37, 20, 3]
    cache = make_cache(dev, 8, H, d, page, seed=91)
    table, lens, starts = tables(held, new, page, 8, dev, seed=92)
    n = sum(new)
    g = torch.Generator().manual_seed(93)
    x = torch.randn((2, n, H, d), generator=g) * torch.pow(2.0, torch.randint(-6, 9, (2, n, 1, 1), generator=g).float())
    special = torch.tensor([math.inf, -math.inf, math.nan, 2.0 ** 108, -2.0 ** 120, 1e-40, 0.0, -0.0])
    for t in (0, 3, 15, 16, 36, 37, 44, 56, 57, 59):
        x[:, t, :, t % 7::9] = special[torch.randint(0, 8, x[:, t, :, t % 7::9].shape, generator=g)]
    x[:, 16:32, 1] = math.nan                           # a whole block of one head
    x[:, 48:50] = 0
    x = x.to(dtype)
    k, v = x[0].to(dev), x[1].to(dev)
    cos, sin = rotation(60, rot // 2) if rot else (None, None)
    pos = np.concatenate([np.arange(p, p + c) for p, c in zip(held, new)])
    kx = x[0].float().numpy()
    with np.errstate(all="ignore"):
        if rot:
            kx = fp32_rotate(kx, cos, sin, pos, False)
        want = expect_append(cache, table.cpu().numpy(), held, new, kx, x[1].float().numpy(), page)
    cache.append(table, lens, None, k, v, *((cos.to(dev), sin.to(dev)) if rot else (None, None)), starts=starts)
    same_codes(cache.k_pages, want[0])
    same_codes(cache.v_pages, want[2])
    assert np.array_equal(cache.k_scale.cpu().numpy().astype(np.float64), want[1])
    assert np.array_equal(cache.v_scale.cpu().numpy().astype(np.float64), want[3])
    assert status()[0] == 0


@pytest.mark.parametrize("out_dtype", [torch.float32, BF])
@pytest.mark.parametrize("held,new", [([40], [1]), ([300, 20], [70, 30]), ([4000], [40])])
def test_outputs_on_16_byte_boundaries(dev, held, new, out_dtype):  # noqa: F811
    d, H, G, page = 128, 2, 4, 64
    cache = make_cache(dev, 70, H, d, page, seed=94)
    table, lens, starts = tables(held, new, page, 70, dev, seed=95)
    n = sum(new)
    q = query(n, H * G, d, 96).to(dev)
    kw = dict(starts=starts, max_new=max(new))
    want, _ = cache.attend(table, lens, q, out_dtype=out_dtype, **kw)
    assert want.data_ptr() % 32 == 0
    off = 16 // want.element_size()
    flat = torch.full((n * H * G * d + 2 * off,), 5.0, dtype=out_dtype, device=dev)
    out = flat[off:off + want.numel()].view_as(want)
    assert out.data_ptr() % 32 == 16
    cache.attend(table, lens, q, out=out, **kw)
    assert torch.equal(out, want) and (flat[:off] == 5).all() and (flat[-off:] == 5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [256, 512, 1024])
def test_large_pages(dev, page, d):  # noqa: F811
    H, G, held, new = 2, 4, [page - 3, 0, 2 * page + 77, 30], [90, 33, 1, 2]
    n = sum(new)
    cache = make_cache(dev, 10, H, d, page, seed=97)
    table, lens, starts = tables(held, new, page, 10, dev, seed=98)
    x = query(n, 2 * H, d, 99, 1.0)
    want = expect_append(cache, table.cpu().numpy(), held, new, x[:, :H].float().numpy(), x[:, H:].float().numpy(), page)
    xd = x.to(dev)
    cache.append(table, lens, None, xd[:, :H], xd[:, H:], starts=starts)
    same_codes(cache.k_pages, want[0])
    same_codes(cache.v_pages, want[2])
    hide_rest(cache, table, held, new, page)
    q = query(n, H * G, d, 100).to(dev)
    for out_dtype in (torch.float32, BF):
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=90, out_dtype=out_dtype, want_lse=True)
        check_attend(out, lse, attend_reference(cache, table, held, new, q, page), out_dtype)
    assert status()[0] == 0


def test_prompts_in_pages_past_four_gigabytes(dev):  # noqa: F811
    from paper_2607_05061_gb300.paged import PagedCache
    H, G, d, page, n, held, new = 8, 2, 128, 64, 70000, 100, 50
    cache = PagedCache.empty(n, H, d, page)
    table = torch.tensor([[n - 1, n - 2, n - 3]], dtype=torch.int32, device=dev)
    k = query(held + new, H, d, 101, 1.0).to(dev)
    zero = torch.zeros(1, dtype=torch.int32, device=dev)
    cache.append(table, zero, None, k, k, starts=torch.tensor([0, held + new], dtype=torch.int32, device=dev))
    q = query(new, H * G, d, 102, 1.0).to(dev)
    out, lse = cache.attend(table, zero + held, q, want_lse=True, max_new=new,
                            starts=torch.tensor([0, new], dtype=torch.int32, device=dev))
    small = PagedCache(*(t[n - 3:].clone() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale)))
    t2 = torch.tensor([[2, 1, 0]], dtype=torch.int32, device=dev)
    check_attend(out, lse, attend_reference(small, t2, [held], [new], q, page), torch.float32)


@pytest.mark.parametrize("out_dtype", [torch.float32, BF])
def test_mixed_batches_in_a_graph_and_on_another_stream(dev, out_dtype):  # noqa: F811
    """Append and attention of prompts among single tokens: three launches that begin early, replayed
    and on a second stream, against the calls one by one."""
    from paper_2607_05061_gb300.paged import PagedCache
    d, H, G, page = 64, 2, 4, 32
    held, new = [700, 3, 90, 1500, 40, 0], [1, 60, 1, 1, 130, 2]
    n = sum(new)
    cache = make_cache(dev, 120, H, d, page, seed=103)
    table, lens, starts = tables([h + 5 * m for h, m in zip(held, new)], new, page, 120, dev, seed=104)
    lens.copy_(torch.tensor(held))
    add = torch.tensor(new, dtype=torch.int32, device=dev)
    rows = query(5 * n, H * G + 2 * H, d, 105, 1.0).to(dev).view(5, n, -1, d)
    twin = PagedCache(*(t.clone() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale)))
    l2 = lens.clone()

    def step(c, at, x, sync):
        q = c.append(table, at, x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:], starts=starts, max_new=130)
        if sync:
            torch.cuda.synchronize()
        out, _ = c.attend(table, at, q, starts=starts, max_new=130, out_dtype=out_dtype)
        if sync:
            torch.cuda.synchronize()
        at += add
        return out
    want = [step(twin, l2, rows[i], True).clone() for i in range(5)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [step(cache, lens, rows[0], False)]
        x = rows[1].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(cache, lens, x, False)
        for i in range(1, 5):
            x.copy_(rows[i])
            graph.replay()
            got.append(out.clone())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(lens, l2) and status()[0] == 0


def test_append_with_idle_places_among_offsets(dev):  # noqa: F811
    """An idle place's rows are passed over: nothing of them is written, rotated queries there keep
    what they held."""
    d, H, page, held, new = 64, 2, 16, [-1, 5, -1, 30, -1], [3, 12, 20, 1, 2]
    n = sum(new)
    cache = make_cache(dev, 8, H, d, page, seed=106)
    table, lens, starts = tables(held, new, page, 8, dev, seed=107)
    x = query(n, 3 * H, d, 108, 1.0)
    want = expect_append(cache, table.cpu().numpy(), held, new, x[:, H:2 * H].float().numpy(), x[:, 2 * H:].float().numpy(), page)
    xd = x.to(dev)
    q_out = torch.full((n, H, d), 3.0, dtype=BF, device=dev)
    cache.append(table, lens, xd[:, :H], xd[:, H:2 * H], xd[:, 2 * H:], starts=starts, q_out=q_out)
    same_codes(cache.k_pages, want[0])
    same_codes(cache.v_pages, want[2])
    live = torch.cat([torch.full((m,), h >= 0) for h, m in zip(held, new)])
    assert torch.equal(q_out.cpu()[live], x[:, :H][live]) and (q_out.cpu()[~live] == 3).all() and status()[0] == 0


@pytest.mark.parametrize("out_dtype", [torch.float32, BF])
@pytest.mark.parametrize("d,G,new", [(128, 4, 1), (64, 4, 1), (128, 7, 2)])
def test_parts_in_groups_of_16(dev, d, G, new, out_dtype):  # noqa: F811
    """One KV head of 40000 positions lies in more than 128 CTAs' parts."""
    page, held = 128, 40000
    n = -(-(held + new) // page)
    cache = make_cache(dev, n, 1, d, page, seed=109)
    table, lens, starts = tables([held], [new], page, n, dev, seed=110)
    q = query(new, G, d, 111).to(dev)
    want = attend_reference(cache, table, [held], [new], q, page)
    first = None
    for _ in range(4):
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=new, out_dtype=out_dtype, want_lse=True)
        check_attend(out, lse, want, out_dtype)
        first = (out.clone(), lse.clone()) if first is None else first
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert status()[0] == 0


@pytest.mark.parametrize("out_dtype", [torch.float32, BF])
@pytest.mark.parametrize("d,n", [(128, 300), (64, 700), (128, 193)])
def test_very_many_sequences(dev, d, n, out_dtype):  # noqa: F811
    """More sequences than a CTA has threads, ragged, every ninth place idle."""
    H, G, page = 1, 4, 16
    r = np.random.default_rng(112)
    held = [-1 if s % 9 == 4 else int(r.integers(0, 200)) for s in range(n)]
    held[7], held[-1] = 1500, 900
    need = sum(-(-(p + 1) // page) for p in held if p >= 0)
    cache = make_cache(dev, need, H, d, page, seed=113)
    table, lens, _ = tables(held, [1] * n, page, need, dev, seed=114)
    hide_rest(cache, table, held, [1] * n, page)
    q = query(n, H * G, d, 115).to(dev)
    want = attend_reference(cache, table, held, [1] * n, q, page)
    for _ in range(2):
        out, lse = cache.attend(table, lens, q, out_dtype=out_dtype, want_lse=True)
        check_attend(out, lse, want, out_dtype)
    assert status()[0] == 0


@pytest.mark.parametrize("out_dtype", [torch.float32, BF])
def test_mixed_batches_of_many_sequences(dev, out_dtype):  # noqa: F811
    """Long sequences beyond the 32nd and the 64th place of a batch of 80, idle ones between."""
    d, H, G, page, n = 64, 2, 4, 16, 80
    r = np.random.default_rng(116)
    held = [-1 if s % 11 == 5 else int(r.integers(0, 120)) for s in range(n)]
    new = [int(r.integers(0, 4)) for _ in range(n)]
    for s, p, k in ((3, 10, 40), (33, 200, 90), (40, 0, 17), (66, 500, 70), (79, 64, 33)):
        held[s], new[s] = p, k
    new[71] = 30                                        # (idle, with rows)
    assert held[71] == -1
    need = sum(-(-(p + k) // page) for p, k in zip(held, new) if p >= 0)
    cache = make_cache(dev, need, H, d, page, seed=117)
    table, lens, starts = tables(held, new, page, need, dev, seed=118)
    hide_rest(cache, table, held, new, page)
    q = query(sum(new), H * G, d, 119).to(dev)
    want = attend_reference(cache, table, held, new, q, page)
    first = None
    for _ in range(3):
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=90, out_dtype=out_dtype, want_lse=True)
        check_attend(out, lse, want, out_dtype)
        first = out.clone() if first is None else first
        assert torch.equal(out, first)
    assert status()[0] == 0
