"""The paged 8-bit cache against its 64-bit oracle: append (rotation, scales, codes, what stays
untouched) and attention (row groups, lengths, masks, NaN, strides, bad tables), on the GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as op

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dev(cuda_device):
    return cuda_device


def status():
    """Status and text of the cache-free calls' record (cleared by reading)."""
    from paper_2607_05061_gb300 import kvpop
    s = kvpop.kvpop_standalone_status(torch.cuda.current_stream().cuda_stream)
    return s, kvpop.kvpop_last_error().decode()


def make_cache(dev, n_pages, H, d, page, seed=0, fill=None):
    """Pages of arbitrary finite bytes (or of `fill`), scales 2^-4 .. 2^3."""
    from paper_2607_05061_gb300.paged import PagedCache
    g = torch.Generator().manual_seed(seed)
    parts = []
    for _ in range(2):
        b = torch.randint(0, 126, (n_pages, H, page, d), generator=g, dtype=torch.int64)
        b += 128 * torch.randint(0, 2, b.shape, generator=g)
        if fill is not None:
            b[:] = fill
        parts.append(b.to(torch.uint8).to(dev).view(F8))
    scales = [torch.pow(2.0, torch.randint(-4, 4, (n_pages, H, page // 16), generator=g).float()).to(dev)
              for _ in range(2)]
    return PagedCache(*parts, *scales)


def tables(held, new, page, n_pages, dev, seed=0, spare=1):
    """Page table (shuffled pages, -1 past the end), lens and starts."""
    need = [-(-(max(p, 0) + n) // page) if p >= 0 else 0 for p, n in zip(held, new)]
    assert sum(need) <= n_pages
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    t = torch.full((len(held), max(need + [1]) + spare), -1, dtype=torch.int32)
    at = 0
    for s, k in enumerate(need):
        t[s, :k] = torch.tensor(ids[at:at + k], dtype=torch.int32)
        at += k
    starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    return t.to(dev), torch.tensor(held, dtype=torch.int32, device=dev), starts.to(dev)


def rotation(n, half):
    ang = np.arange(n)[:, None] * 10000.0 ** (-np.arange(half) / half)
    return torch.tensor(np.cos(ang)).float(), torch.tensor(np.sin(ang)).float()


# ------------------------------------------------------------------ append
def fp32_rotate(x, cos, sin, pos, interleaved):
    """The documented fp32 rotation of x [n][heads][d] (numpy, each operation rounded once)."""
    y = x.copy()
    half = cos.shape[1]
    c, s = cos[pos][:, None].numpy(), sin[pos][:, None].numpy()
    ia = np.arange(0, 2 * half, 2) if interleaved else np.arange(half)
    ib = ia + 1 if interleaved else ia + half
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def expect_append(cache, table, held, new, k, v, page):
    """Pages and scales after an append of k, v (fp32 [n][H][d], rotated), from the oracle."""
    out = []
    for pages, scale, x in ((cache.k_pages, cache.k_scale, k), (cache.v_pages, cache.v_scale, v)):
        b, sc = pages.view(torch.uint8).cpu().numpy().copy(), scale.cpu().numpy().astype(np.float64)
        at = 0
        for s, (p, n) in enumerate(zip(held, new)):
            done = 0
            while p >= 0 and done < n:
                pos = p + done
                m = min(16 - pos % 16, n - done)
                pg, blk, row = int(table[s, pos // page]), pos % page // 16, pos % 16
                for h in range(b.shape[1]):
                    sc[pg, h, blk] = op.append_tokens(b[pg, h, blk * 16:blk * 16 + 16], sc[pg, h, blk], row,
                                                      x[at + done:at + done + m, h].astype(np.float64))
                done += m
            at += n
        out += [b, sc]
    return out


def same_codes(got, want):
    got = got.view(torch.uint8).cpu().numpy()
    nan = (got & 127) == 127
    assert np.array_equal(nan, (want & 127) == 127)
    assert np.array_equal(got[~nan], want[~nan])


CASES = [
    # dtype, d, H, G, page, rot, interleaved, held, new (None: one token each, no starts)
    ("bf16", 128, 2, 2, 16, 128, False, [0, 5, 15, 16, 31, 100], None),
    ("f32", 64, 3, 1, 32, 64, False, [0, 1, 47], None),
    ("bf16", 64, 1, 3, 64, 32, True, [7, 63, 64], None),
    ("bf16", 128, 2, 4, 64, 128, False, [0, 3, 70, 15], [33, 1, 0, 130]),
    ("f32", 128, 1, 1, 16, 48, True, [9], [75]),
    ("f32", 64, 2, 2, 128, 16, False, [120, 0, 31], [17, 16, 1]),
    ("bf16", 64, 5, 1, 16, 0, False, [2, 14], [15, 2]),
]


@pytest.mark.parametrize("case", CASES)
def test_append(dev, case):
    dtype, d, H, G, page, rot, inter, held, new = case
    counts = new or [1] * len(held)
    cache = make_cache(dev, 24, H, d, page)
    table, lens, starts = tables(held, counts, page, 24, dev)
    n = sum(counts)
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((n, H * G + 2 * H, d), generator=g) * torch.pow(2.0, torch.randint(-6, 9, (n, 1, 1), generator=g).float())
    qkv = qkv.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    dq = qkv.to(dev)
    q, k, v = dq[:, :H * G], dq[:, H * G:H * G + H], dq[:, H * G + H:]     # columns of one tensor's rows
    cos, sin = rotation(300, rot // 2) if rot else (None, None)
    pos = np.concatenate([np.arange(p, p + c) for p, c in zip(held, counts)]).astype(np.int64)
    x = qkv.float().numpy()
    turn = lambda y: fp32_rotate(y, cos, sin, pos, inter) if rot else y  # noqa: E731
    want = expect_append(cache, table.cpu().numpy(), held, counts, turn(x[:, H * G:H * G + H]), x[:, H * G + H:], page)
    got = cache.append(table, lens, q, k, v, *((cos.to(dev), sin.to(dev)) if rot else (None, None)),
                       starts=None if new is None else starts, interleaved=inter)
    same_codes(cache.k_pages, want[0])
    same_codes(cache.v_pages, want[2])
    assert np.array_equal(cache.k_scale.cpu().numpy().astype(np.float64), want[1])
    assert np.array_equal(cache.v_scale.cpu().numpy().astype(np.float64), want[3])
    assert torch.equal(got.cpu(), torch.from_numpy(turn(x[:, :H * G])).bfloat16())
    # the fp32 rotation itself: two products and a sum, each rounded once
    if rot:
        for i in range(0, n, 7):
            y = op.rotate(x[i, 0], cos[pos[i]].numpy(), sin[pos[i]].numpy(), inter)
            assert np.abs(turn(x[:, :1])[i, 0] - y).max() <= 3 * 2.0 ** -24 * 2 * np.abs(x[i, 0]).max()
    assert status()[0] == 0


def test_scales_that_grow_token_by_token(dev):
    """One token at a time with growing, shrinking, zero and special values, over a page's stale
    NaN: each step as the oracle's, rows past the last token untouched."""
    d, H, page = 64, 1, 16
    cache = make_cache(dev, 3, H, d, page, fill=127)
    table = torch.tensor([[2, 0]], dtype=torch.int32, device=dev)
    g = torch.Generator().manual_seed(4)
    x = torch.randn((20, H, d), generator=g) * torch.pow(2.0, torch.tensor([0., 3, -9, 3, 4, 20, 19, 21, -30, 0, 1, 2, 25, 0,
                                                                            26, 3, 0, 1, -2, 5]))[:, None, None]
    x[1, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, -0.0])
    x[4] = 0.0
    x[16] = 0.0                                    # a block that begins with nothing but zeros
    x[6, 0, 5] = 2.0 ** 108                        # too large for any scale
    x[7, 0, 6] = 1e-40                             # subnormal
    codes = np.full((32, d), 127, np.uint8)
    scale = [0.0, 0.0]
    for i in range(20):
        cache.append(table, torch.tensor([i], dtype=torch.int32, device=dev), None, x[i:i + 1].to(dev), x[i:i + 1].to(dev))
        b = i // 16
        scale[b] = op.append_token(codes[16 * b:16 * b + 16], scale[b], i % 16, x[i, 0].double().numpy())
        for pages, sc in ((cache.k_pages, cache.k_scale), (cache.v_pages, cache.v_scale)):
            got = pages.view(torch.uint8).cpu().numpy()[[2, 0], 0].reshape(32, d)
            nan = (codes & 127) == 127
            assert np.array_equal((got & 127) == 127, nan)
            assert np.array_equal(got[~nan], codes[~nan])
            assert sc[2, 0, 0].item() == scale[0] and (b == 0 or sc[0, 0, 0].item() == scale[1])
    assert (cache.k_pages.view(torch.uint8)[1] == 127).all()


def test_append_passes_over_idle_places_and_records_bad_tables(dev):
    d, H, page = 128, 2, 16
    bf = torch.bfloat16
    k = torch.randn(4, H, d, device=dev, dtype=bf)
    cos, sin = (t.to(dev) for t in rotation(40, 64))

    def run(lens, table, cos=cos, sin=sin):
        cache = make_cache(dev, 6, H, d, page)
        before = [t.clone() for t in (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scale,
                                      cache.v_scale)]
        cache.append(torch.tensor(table, dtype=torch.int32, device=dev),
                     torch.tensor(lens, dtype=torch.int32, device=dev), None, k, k, cos, sin)
        after = (cache.k_pages.view(torch.uint8), cache.v_pages.view(torch.uint8), cache.k_scale, cache.v_scale)
        return status(), [sorted(set((a != b).flatten(1).any(1).nonzero().flatten().tolist()))
                          for a, b in zip(after, before)]

    good = [[0, 1], [2, 3], [4, 5], [-1, -1]]
    (st, _), pages = run([3, -1, 20, -1], good)
    assert st == 0 and pages[0] == [0, 5]
    (st, _), pages = run([3, 16, 20, -1], [[0, 1], [2, 6], [4, -1], [-1, -1]])     # a page past the pool, a hole
    assert st == 6 and pages[0] == [0]
    (st, _), pages = run([32, 4, -1, -1], good)                                    # past the table
    assert st == 6 and pages[0] == [2]
    (st, _), pages = run([2 ** 31 - 1, 4, -1, -1], good)
    assert st == 6 and pages[0] == [2]
    (st, _), pages = run([20, 3, -1, -1], good, cos[:20], sin[:20])                # past the rotation table
    assert st == 6 and pages[0] == [2]
    assert status()[0] == 0


def test_append_with_offsets_that_do_not_ascend(dev):
    cache = make_cache(dev, 8, 1, 64, 16)
    k = torch.randn(20, 1, 64, device=dev)
    table = torch.arange(8, dtype=torch.int32, device=dev).view(2, 4)
    lens = torch.zeros(2, dtype=torch.int32, device=dev)
    for starts in ([0, 30, 20], [-5, 10, 20], [0, 12, 4], [2 ** 31 - 1, -2 ** 31, 7]):
        cache.append(table, lens, None, k, k, starts=torch.tensor(starts, dtype=torch.int32, device=dev))
        assert status()[0] == 6


# ------------------------------------------------------------------ attention
def attend_reference(cache, table, held, new, q, page):
    """(y, lse, tolerance of the weights, largest |v|) per token and head, fp64 on the CPU."""
    H, d = cache.H, cache.d
    G = q.shape[1] // H
    kb, vb = (op.E4M3[t.view(torch.uint8).cpu().numpy()] for t in (cache.k_pages, cache.v_pages))
    kb = kb * np.repeat(cache.k_scale.cpu().numpy().astype(np.float64), 16, -1)[..., None]
    vb = vb * np.repeat(cache.v_scale.cpu().numpy().astype(np.float64), 16, -1)[..., None]
    qd = q.double().cpu().numpy()
    y, lse = np.zeros(qd.shape), np.full(qd.shape[:2], -math.inf)
    eps, top = np.zeros(qd.shape[:2]), np.zeros(qd.shape[:2])
    at = 0
    tb = table.cpu().numpy()
    for s, (p, n) in enumerate(zip(held, new)):
        if p >= 0:
            ids = tb[s, :-(-(p + n) // page)]
            for h in range(H):
                K, V = kb[ids, h].reshape(-1, d), vb[ids, h].reshape(-1, d)
                for i in range(n):
                    t = p + i + 1
                    for g in range(G):
                        r = (at + i, h * G + g)
                        y[r], lse[r] = op.attend(qd[r], K[:t], V[:t])
                        eps[r] = (np.abs(K[:t]) @ np.abs(qd[r])).max() / math.sqrt(d)
                        top[r] = np.abs(V[:t]).max()
        at += n
    return y, lse, eps, top


def check_attend(got, lse, want, out_dtype):
    """fp32 sums of the logits (2^-21 of the sum of magnitudes), 2^-20 for exponentials and sums,
    the weights' 22 or 11 bits, and the rounding of the result."""
    y, wl, a, top = want
    eps = 2.0 ** -21 * a + 2.0 ** -20
    w = 2.0 ** -21 if out_dtype == torch.float32 else 2.0 ** -11
    tol = (2 * (eps + w) * top)[..., None] + (2.0 ** -23 if out_dtype == torch.float32 else 2.0 ** -8) * np.abs(y)
    d = np.abs(got.double().cpu().numpy() - y)
    assert (d <= tol).all(), (d / np.maximum(tol, 1e-300)).max()
    live = np.isfinite(wl)
    gl = lse.double().cpu().numpy()
    assert np.array_equal(np.isfinite(gl), live) and (gl[~live] == -math.inf).all()
    assert (np.abs(gl[live] - wl[live]) <= (2 * eps + 2.0 ** -22 * np.abs(wl))[live]).all()


ATTEND = [
    # d, H, G, page, held, new (None: one token each)
    (128, 2, 4, 16, [0, 1, 14, 15, 16, 17, 31, 200], None),
    (128, 1, 1, 64, [1029], None),
    (64, 3, 2, 32, [0, 33, 511], None),
    (128, 2, 8, 64, [130, 7], None),
    (64, 2, 7, 16, [77, 300, 0], None),
    (128, 1, 16, 16, [40, 3], None),                # two groups of 8 rows
    (64, 1, 13, 16, [40, 3], None),
    (128, 1, 40, 16, [50], None),                   # more than 32 rows for one token
    (128, 2, 4, 64, [100, 0, 15, 64], [5, 3, 1, 4]),
    (64, 2, 3, 16, [9, 31], [2, 6]),
    (128, 2, 1, 32, [17, 250], [9, 16]),
    (64, 1, 4, 16, [0], [8]),
    (128, 1, 4, 128, [5, 200], [40, 19]),           # longer than a row group
    (64, 2, 2, 64, [0, 3, 90], [150, 1, 33]),
    (128, 1, 4, 64, [0], [17]),                     # one row more than a short sequence has
    (128, 2, 4, 64, [130, 0, 700], [64, 65, 129]),  # 256 rows, one token more, and a third tile
    (128, 1, 7, 16, [3, 511], [37, 80]),            # tiles that cut a token's heads
    (64, 1, 1, 128, [250], [600]),
    (128, 1, 8, 32, [1200], [33]),                  # more blocks than the ring holds
    (64, 3, 4, 16, [0, 5, 20, 7], [40, 2, 0, 90]),  # short and long ones in one call
]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", ATTEND)
def test_attend(dev, case, out_dtype):
    d, H, G, page, held, new = case
    counts = new or [1] * len(held)
    cache = make_cache(dev, 40, H, d, page, seed=2)
    table, lens, starts = tables(held, counts, page, 40, dev, seed=3)
    hide_rest(cache, table, held, counts, page)
    q = (torch.randn((sum(counts), H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, starts=None if new is None else starts, out_dtype=out_dtype,
                            max_new=max(counts), want_lse=True)
    check_attend(out, lse, attend_reference(cache, table, held, counts, q, page), out_dtype)
    assert status()[0] == 0
    again, lse2 = cache.attend(table, lens, q, starts=None if new is None else starts, out_dtype=out_dtype,
                               max_new=max(counts), want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def hide_rest(cache, table, held, counts, page):
    """NaN in every row that no sequence holds."""
    keep = torch.zeros(cache.k_pages.shape[:1] + (page,), dtype=torch.bool)
    tb = table.cpu()
    for s, (p, n) in enumerate(zip(held, counts)):
        for t in range(max(p, 0) + n if p >= 0 else 0):
            keep[tb[s, t // page], t % page] = True
    for pages in (cache.k_pages, cache.v_pages):
        b = pages.view(torch.uint8)
        b[(~keep).to(b.device)[:, None].expand(b.shape[:3])] = 127


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_attend_long_rows_over_many_parts(dev, out_dtype):
    """Contexts cut over many CTAs, ragged, and one sequence whose parts other sequences share."""
    held, d, H, G, page = [5003, 17, 2500, 0, 777], 128, 2, 4, 64
    cache = make_cache(dev, 160, H, d, page, seed=6)
    table, lens, _ = tables(held, [1] * 5, page, 160, dev, seed=7)
    q = (torch.randn((5, H * G, d), generator=torch.Generator().manual_seed(8)) * 0.02).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, out_dtype=out_dtype, want_lse=True)
    check_attend(out, lse, attend_reference(cache, table, held, [1] * 5, q, page), out_dtype)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_long_tiles_cut_into_parts(dev, d, out_dtype):
    """Few tiles over many positions: each tile's positions are cut, one sequence's last part holds
    nothing that its first rows see, and short sequences run beside them."""
    held, new, H, G, page = [4000, 1500, 0, 90, -1], [40, 130, 300, 1, 2], 1, 4, 64
    cache = make_cache(dev, 110, H, d, page, seed=18)
    table, lens, starts = tables(held, new, page, 110, dev, seed=19)
    hide_rest(cache, table, held, new, page)
    cache.v_pages.view(torch.uint8)[int(table[0, 4010 // page]), 0, 4010 % page, 11] = 127    # token 10's
    q = (torch.randn((sum(new), H * G, d), generator=torch.Generator().manual_seed(8)) * 0.02).bfloat16().to(dev)
    want = attend_reference(cache, table, held, new, q, page)
    y, bad = want[0], np.isnan(want[0])
    assert not bad[:10].any() and bad[10:40, :, 11].all() and bad.sum() == 30 * G
    for _ in range(2):
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=300, out_dtype=out_dtype, want_lse=True)
        got = out.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), bad)
        clean = torch.from_numpy(np.where(bad, 0, got))
        top = np.where(np.isnan(want[3]), np.nanmax(want[3]), want[3])
        check_attend(clean, lse, (np.where(bad, 0, y), want[1], want[2], top), out_dtype)
    assert status()[0] == 0


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,G,new", [(128, 4, [1, 1, 1]), (64, 7, [1, 3, 1]), (128, 16, [2, 1, 1])])
def test_few_heads_over_many_positions(dev, d, G, new, out_dtype):
    """A KV head's positions lie in the parts of very many CTAs, which join in groups; a second
    sequence ends inside a part, a third is short."""
    held, H, page = [9000, 5003, 70], 1, 128
    cache = make_cache(dev, 120, H, d, page, seed=28)
    table, lens, starts = tables(held, new, page, 120, dev, seed=29)
    hide_rest(cache, table, held, new, page)
    q = (torch.randn((sum(new), H * G, d), generator=torch.Generator().manual_seed(9)) * 0.02).bfloat16().to(dev)
    want = attend_reference(cache, table, held, new, q, page)
    first = None
    for _ in range(3):
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=3, out_dtype=out_dtype, want_lse=True)
        check_attend(out, lse, want, out_dtype)
        first = out.clone() if first is None else first
        assert torch.equal(out, first)
    assert status()[0] == 0


def test_idle_places_and_sequences_without_tokens(dev):
    d, H, G, page = 128, 2, 4, 16
    cache = make_cache(dev, 16, H, d, page, seed=9)
    for held, new, most in (([-1, 20, -1, 5, 0], [3, 0, 1, 2, 1], 3), ([-1, 20, -1, 5, 0], [30, 0, 1, 40, 1], 40)):
        table, lens, starts = tables(held, new, page, 16, dev)
        q = (torch.randn((sum(new), H * G, d)) * 0.02).bfloat16().to(dev)
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=most, want_lse=True)
        check_attend(out, lse, attend_reference(cache, table, held, new, q, page), torch.float32)
        n = new[0] + 1
        assert (out[:n] == 0).all() and (lse[:n] == -math.inf).all() and status()[0] == 0


def test_scales_far_apart(dev):
    """Blocks whose value scales differ by 2^40, and keys of very different size."""
    d, H, G, page, held = 64, 1, 4, 16, [95]
    cache = make_cache(dev, 6, H, d, page, seed=10)
    cache.v_scale.copy_(torch.tensor([2.0 ** e for e in (-20, 20, 0, -40, 7, 3)], device=dev).view(6, 1, 1))
    cache.k_scale.copy_(torch.tensor([2.0 ** e for e in (-10, -3, -8, -4, -20, -90)], device=dev).view(6, 1, 1))
    for held, new in (([95], [1]), ([63], [33])):
        table, lens, starts = tables(held, new, page, 6, dev)
        q = (torch.randn((new[0], G, d), generator=torch.Generator().manual_seed(2)) * 0.05).bfloat16().to(dev)
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=new[0], want_lse=True)
        check_attend(out, lse, attend_reference(cache, table, held, new, q, page), torch.float32)


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -30, 2.0 ** 30])
def test_queries_of_any_size(dev, size):
    d, H, G, page, held = 128, 1, 2, 16, [40]
    cache = make_cache(dev, 4, H, d, page, seed=11)
    cache.k_scale.fill_(2.0 ** -34 if size > 1 else 2.0 ** 26 if size > 2.0 ** -40 else 2.0 ** 90)
    table, lens, _ = tables(held, [1], page, 4, dev)
    q = (torch.randn((1, G, d), generator=torch.Generator().manual_seed(2)) * size).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, want_lse=True)
    check_attend(out, lse, attend_reference(cache, table, held, [1], q, page), torch.float32)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [1, 6, 50])
def test_logits_that_rise_and_fall_along_the_keys(dev, new, out_dtype):
    """The running base moves often: key scales grow block by block, then shrink."""
    d, H, G, page, held = 128, 1, 4, 32, [700]
    cache = make_cache(dev, 24, H, d, page, seed=16)
    table, lens, starts = tables(held, [new], page, 24, dev)
    n = -(-(held[0] + new) // page)
    for i in range(n):
        cache.k_scale[int(table[0, i])] = 2.0 ** (-6 + min(i, n - 1 - i) * 0.25 // 1)
    q = (torch.randn((new, G, d), generator=torch.Generator().manual_seed(2)) * 0.05).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, starts=starts, max_new=new, out_dtype=out_dtype, want_lse=True)
    check_attend(out, lse, attend_reference(cache, table, held, [new], q, page), out_dtype)


def test_outputs_do_not_rest_on_max_new(dev):
    d, H, G, page, held, new = 128, 2, 4, 64, [40, 9], [30, 2]
    cache = make_cache(dev, 8, H, d, page, seed=17)
    table, lens, starts = tables(held, new, page, 8, dev)
    q = (torch.randn((32, H * G, d)) * 0.02).bfloat16().to(dev)
    want = attend_reference(cache, table, held, new, q, page)
    for most in (1, 2, 4, 8, 30, 10 ** 9, None):
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=most, want_lse=True)
        check_attend(out, lse, want, torch.float32)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [4, 40])
def test_nan_reaches_the_rows_that_see_it_and_no_other(dev, new, out_dtype):
    """A NaN value of a new token: NaN in that column for the tokens from it on, nothing for the
    ones before; a NaN key: whole rows from it on."""
    d, H, G, page, held = 128, 2, 2, 16, [21]
    for part in ("v", "k"):
        cache = make_cache(dev, 8, H, d, page, seed=12)
        table, lens, starts = tables(held, [new], page, 8, dev)
        q = (torch.randn((new, H * G, d)) * 0.02).bfloat16().to(dev)
        clean, clean_lse = cache.attend(table, lens, q, starts=starts, max_new=new, out_dtype=out_dtype, want_lse=True)
        at = 21 + 2
        pages = cache.v_pages if part == "v" else cache.k_pages
        pages.view(torch.uint8)[int(table[0, at // page]), 1, at % page, 37] = 127
        out, lse = cache.attend(table, lens, q, starts=starts, max_new=new, out_dtype=out_dtype, want_lse=True)
        bad = torch.zeros_like(out, dtype=torch.bool)
        if part == "v":
            bad[2:, G:, 37] = True
        else:
            bad[2:, G:] = True
        assert torch.equal(torch.isnan(out), bad)
        near = (out.float() - clean.float()).abs() <= 2.0 ** -7 * clean.float().abs() + 1e-5
        assert near[~bad].all()
        if part == "v":
            assert torch.equal(lse, clean_lse)


def test_a_bad_page_is_left_out_and_recorded(dev):
    d, H, G, page, held = 64, 2, 2, 16, [60]
    cache = make_cache(dev, 5, H, d, page, seed=13)
    q = (torch.randn((1, H * G, d)) * 0.02).bfloat16().to(dev)
    lens = torch.tensor(held, dtype=torch.int32, device=dev)
    for bad in (-1, 5, 2 ** 31 - 1):
        table = torch.tensor([[0, bad, 2, 3]], dtype=torch.int32, device=dev)
        out, _ = cache.attend(table, lens, q)
        assert status()[0] == 6
        short = torch.tensor([[0, 2, 3]], dtype=torch.int32, device=dev)
        want, _ = cache.attend(short, lens - 16, q)
        assert torch.allclose(out, want, rtol=1e-5, atol=1e-5) and status()[0] == 0
    out, _ = cache.attend(torch.tensor([[0, 1]], dtype=torch.int32, device=dev), lens, q)   # past the table
    assert status()[0] == 6
    want, _ = cache.attend(torch.tensor([[0, 1]], dtype=torch.int32, device=dev), lens * 0 + 31, q)
    assert torch.equal(out, want) and status()[0] == 0


def test_strided_queries_and_tables(dev):
    d, H, G, page, held = 64, 2, 3, 16, [30, 45]
    cache = make_cache(dev, 8, H, d, page, seed=14)
    table, lens, _ = tables(held, [1, 1], page, 8, dev, spare=3)
    q = (torch.randn((2, H * G, d)) * 0.02).bfloat16().to(dev)
    want, _ = cache.attend(table, lens, q)
    wide = torch.zeros((2, 3, H * G, d), dtype=torch.bfloat16, device=dev)
    wide[:, 1] = q
    assert torch.equal(cache.attend(table, lens, wide[:, 1])[0], want)
    heads_first = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(cache.attend(table[:, :4], lens, heads_first)[0], want)


def test_pages_past_four_gigabytes(dev):
    """The pool is 4.6 GB and the sequence lies in its last pages."""
    from paper_2607_05061_gb300.paged import PagedCache
    H, d, page, n = 8, 128, 64, 70000
    cache = PagedCache.empty(n, H, d, page)
    held = 150
    table = torch.tensor([[n - 1, n - 2, n - 3]], dtype=torch.int32, device=dev)
    k = torch.randn((held + 1, H, d), generator=torch.Generator().manual_seed(1)).bfloat16().to(dev)
    zero = torch.zeros(1, dtype=torch.int32, device=dev)
    cache.append(table, zero, None, k, k, starts=torch.tensor([0, held + 1], dtype=torch.int32, device=dev))
    q = torch.randn((1, H, d), generator=torch.Generator().manual_seed(2)).bfloat16().to(dev)
    out, lse = cache.attend(table, zero + held, q, want_lse=True)
    small = PagedCache(*(t[n - 3:].clone() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale)))
    t2 = torch.tensor([[2, 1, 0]], dtype=torch.int32, device=dev)
    check_attend(out, lse, attend_reference(small, t2, [held], [1], q, page), torch.float32)
    assert (cache.k_pages.view(torch.uint8)[:n - 3] == 0).all()


def test_another_stream_and_a_captured_graph(dev):
    d, H, G, page = 128, 2, 4, 16
    cache = make_cache(dev, 20, H, d, page, seed=15)
    held = [10, 40]
    table, lens, _ = tables([60, 60], [1, 1], page, 20, dev)
    lens.copy_(torch.tensor(held))
    cos, sin = (t.to(dev) for t in rotation(100, 64))
    rows = torch.randn((8, 2, H * G + 2 * H, d), generator=torch.Generator().manual_seed(3)).bfloat16().to(dev)

    def step(cache, lens, x):
        q = cache.append(table, lens, x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:], cos, sin)
        out, _ = cache.attend(table, lens, q)
        lens += 1
        return out
    from paper_2607_05061_gb300.paged import PagedCache
    copy = PagedCache(*(t.clone() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale)))
    l2 = lens.clone()
    want = [step(copy, l2, rows[i]).clone() for i in range(8)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [step(cache, lens, rows[i]) for i in range(3)]
        x = rows[3].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(cache, lens, x)
        for i in range(3, 8):
            x.copy_(rows[i])
            graph.replay()
            got.append(out.clone())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(lens, l2) and status()[0] == 0
