"""Append of tokens whose positions are given: on one axis, on several, out of the tables, captured."""
import numpy as np
import pytest
import torch

from test_gpu_paged import dev, expect_append, make_cache, rotation, same_codes, status, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def turn(x, cos, sin, pos, axes, interleaved):
    """The documented fp32 rotation of x [n][heads][d]: pair j by row pos[i][axes[j]]."""
    y, half = x.copy(), cos.shape[1]
    rows = pos[:, list(axes)]                                       # [n][half]
    c, s = (t.numpy()[rows, np.arange(half)][:, None] for t in (cos, sin))
    ia = np.arange(0, 2 * half, 2) if interleaved else np.arange(half)
    ib = ia + 1 if interleaved else ia + half
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def third(half):
    return [0] * (half // 4) + [1] * (half // 2 - half // 4) + [2] * (half - half // 2)


CASES = [
    # dtype, d, H, G, page, rot, interleaved, held, new (None: one token each), axes (None: one axis, 1-D)
    ("bf16", 128, 2, 2, 16, 128, False, [0, 5, 15, 16, 31, 100], None, None),
    ("f32", 64, 3, 1, 32, 64, False, [0, 1, 47], None, third(32)),
    ("bf16", 64, 1, 3, 64, 32, True, [7, 63, 64], None, third(16)),
    ("bf16", 128, 2, 4, 64, 128, False, [0, 3, 70, 15], [33, 1, 0, 130], third(64)),
    ("f32", 128, 1, 1, 16, 48, True, [9], [75], [j % 3 for j in range(24)]),       # axes that change with every pair
    ("bf16", 128, 1, 5, 16, 128, False, [2, 8], [40, 17], [j % 4 for j in range(64)]),
    ("f32", 64, 2, 2, 128, 16, False, [120, 0, 31], [17, 16, 1], [1] * 8),          # an axis that no pair uses
    ("bf16", 64, 5, 1, 16, 64, False, [2, 14], [15, 2], None),
]


@pytest.mark.parametrize("case", CASES)
def test_append_at_positions(dev, case):
    dtype, d, H, G, page, rot, inter, held, new, axes = case
    counts = new or [1] * len(held)
    cache = make_cache(dev, 24, H, d, page)
    table, lens, starts = tables(held, counts, page, 24, dev)
    n = sum(counts)
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((n, H * G + 2 * H, d), generator=g) * torch.pow(2.0, torch.randint(-6, 9, (n, 1, 1), generator=g).float())
    qkv = qkv.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    dq = qkv.to(dev)
    cos, sin = rotation(300, rot // 2)
    n_axes = 1 if axes is None else max(axes) + 1
    pos = torch.randint(0, 300, (n, n_axes), generator=g, dtype=torch.int32)
    pos[0], pos[-1] = 0, 299
    x = qkv.float().numpy()
    do = lambda y: turn(y, cos, sin, pos.long().numpy(), axes or [0] * (rot // 2), inter)  # noqa: E731
    want = expect_append(cache, table.cpu().numpy(), held, counts, do(x[:, H * G:H * G + H]), x[:, H * G + H:], page)
    got = cache.append(table, lens, dq[:, :H * G], dq[:, H * G:H * G + H], dq[:, H * G + H:], cos.to(dev), sin.to(dev),
                       starts=None if new is None else starts, interleaved=inter,
                       positions=(pos[:, 0] if axes is None else pos).contiguous().to(dev), axes=axes)
    same_codes(cache.k_pages, want[0])
    same_codes(cache.v_pages, want[2])
    assert np.array_equal(cache.k_scale.cpu().numpy().astype(np.float64), want[1])
    assert np.array_equal(cache.v_scale.cpu().numpy().astype(np.float64), want[3])
    assert torch.equal(got.cpu(), torch.from_numpy(do(x[:, :H * G])).bfloat16())
    assert status()[0] == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [None, [21, 40]])
def test_places_as_positions_are_the_plain_append(dev, d, new):
    """Positions that are the tokens' places give bit for bit what is given without them."""
    held, H, G, page = [30, 7], 2, 3, 32
    counts = new or [1, 1]
    table, lens, starts = tables(held, counts, page, 8, dev)
    n = sum(counts)
    x = torch.randn((n, H * G + 2 * H, d), generator=torch.Generator().manual_seed(2)).bfloat16().to(dev)
    cos, sin = (t.to(dev) for t in rotation(100, d // 2))
    pos = torch.tensor(np.concatenate([np.arange(p, p + c) for p, c in zip(held, counts)]), dtype=torch.int32, device=dev)
    got = []
    for kw in ({}, dict(positions=pos), dict(positions=pos[:, None].contiguous(), axes=bytes(d // 2)),
               dict(positions=torch.stack([pos, pos * 0, pos], 1).contiguous(), axes=[0, 2] * (d // 4))):
        cache = make_cache(dev, 8, H, d, page)
        q = cache.append(table, lens, x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:], cos, sin,
                         starts=None if new is None else starts, **kw)
        got.append([q, cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scale, cache.v_scale])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("new", [None, [5, 20]])
def test_positions_out_of_the_tables(dev, new):
    """Such tokens are recorded and left out, in whichever axis: the others are as without them."""
    held, H, G, page, d = [3, 12], 1, 2, 16, 64
    counts = new or [1, 1]
    table, lens, starts = tables(held, counts, page, 8, dev)
    n = sum(counts)
    x = torch.randn((n, H * G + 2 * H, d), generator=torch.Generator().manual_seed(3))
    cos, sin = rotation(50, d // 2)
    good = torch.randint(0, 50, (n, 2), generator=torch.Generator().manual_seed(4), dtype=torch.int32)
    axes = [0] * 32                                                 # the second axis turns no pair
    for where, bad in ((0, -1), (0, 50), (n - 1, 2 ** 31 - 1), (n - 1, -2 ** 31)):
        for axis in (0, 1):
            pos = good.clone()
            pos[where, axis] = bad
            cache, ref = make_cache(dev, 8, H, d, page), make_cache(dev, 8, H, d, page)
            before = cache.k_pages.view(torch.uint8).clone()
            q_out = torch.full((n, H * G, d), 7.0, dtype=torch.bfloat16, device=dev)
            xd = x.to(dev)
            cache.append(table, lens, xd[:, :H * G], xd[:, H * G:H * G + H], xd[:, H * G + H:], cos.to(dev), sin.to(dev),
                         starts=None if new is None else starts, positions=pos.to(dev), axes=axes, q_out=q_out)
            assert status()[0] == 6
            # the same tokens with a zero key and value there count nothing in their block's scale
            keep = torch.ones(n, dtype=torch.bool)
            keep[where] = False
            xz = x.clone()
            xz[where] = 0
            xz = xz.to(dev)
            want = ref.append(table, lens, xz[:, :H * G], xz[:, H * G:H * G + H], xz[:, H * G + H:], cos.to(dev),
                              sin.to(dev), starts=None if new is None else starts, positions=good.to(dev), axes=axes)
            assert status()[0] == 0
            assert torch.equal(q_out.cpu()[keep], want.cpu()[keep]) and (q_out[where] == 7).all()
            s = 0 if where < counts[0] else 1
            place = held[s] + where - (0 if s == 0 else counts[0])
            page_id, row = int(table[s, place // page]), place % page
            a, b = cache.k_pages.view(torch.uint8).clone(), ref.k_pages.view(torch.uint8).clone()
            assert torch.equal(a[page_id, :, row], before[page_id, :, row])
            a[page_id, :, row] = b[page_id, :, row] = 0
            assert torch.equal(a, b)
            if not (new is None and place % 16 == 0):
                assert torch.equal(cache.k_scale, ref.k_scale)


def test_captured_append_reads_positions_anew(dev):
    held, H, G, page, d = [40, 3, 17], 2, 2, 16, 128
    table, lens, _ = tables(held, [1] * 3, page, 16, dev)
    x = torch.randn((3, H * G + 2 * H, d), generator=torch.Generator().manual_seed(5)).bfloat16().to(dev)
    cos, sin = (t.to(dev) for t in rotation(90, d // 2))
    pos = torch.tensor([[1, 2, 3], [4, 5, 6], [7, 8, 9]], dtype=torch.int32, device=dev)
    axes = bytes(third(64))
    cache, plain = make_cache(dev, 16, H, d, page), make_cache(dev, 16, H, d, page)
    args = (x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:], cos, sin)
    q_out = torch.empty((3, H * G, d), dtype=torch.bfloat16, device=dev)
    cache.append(table, lens, *args, positions=pos, axes=axes, q_out=q_out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(table, lens, *args, positions=pos, axes=axes, q_out=q_out)
    pos += 33
    graph.replay()
    want = plain.append(table, lens, *args, positions=pos, axes=axes)
    assert torch.equal(q_out, want)
    assert status()[0] == 0
