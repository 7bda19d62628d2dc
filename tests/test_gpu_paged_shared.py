"""Attention over shared prefixes against 64 bits: groups of every kind, lengths, masks, parts of the
positions and their joins, bad groups, capture and streams."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import attend_reference, check_attend, dev, hide_rest, make_cache, status  # noqa: F401

pytestmark = pytest.mark.gpu


def shared_tables(first, prefix, held, new, page, dev, seed=0):
    """A table in which the members of a group have the pages of its prefix in common (whole pages;
    tokens of a page that the prefix ends in are each sequence's own copy), lens, starts."""
    n = len(held)
    common = [0] * n
    lead = list(range(n))
    for g, p in enumerate(prefix):
        for s in range(first[g], first[g + 1]):
            common[s], lead[s] = p // page, first[g]
    need = [-(-(max(p, 0) + k) // page) if p >= 0 else 0 for p, k in zip(held, new)]
    total = sum(need) + sum(prefix) // page + 4
    ids = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
    pages = {}
    t = torch.full((n, max(need + [1]) + 1), -1, dtype=torch.int32)
    for s in range(n):
        for i in range(need[s]):
            key = (lead[s], i) if i < common[s] else (s, i, "own")
            if key not in pages:
                pages[key] = ids.pop()
            t[s, i] = pages[key]
    starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    return t.to(dev), torch.tensor(held, dtype=torch.int32, device=dev), starts.to(dev), total


def same_prefix(cache, table, first, prefix, held, page):
    """The rest of a prefix, behind its whole pages: every member's copy of the first one's rows."""
    for g, p in enumerate(prefix):
        live = [s for s in range(first[g], first[g + 1]) if held[s] >= 0]
        rest = p - p // page * page
        if len(live) < 2 or rest == 0:
            continue
        i = p // page
        for s in live[1:]:
            if held[s] < p:
                continue
            a, b = int(table[live[0], i]), int(table[s, i])
            if a < 0 or b < 0:
                continue
            for pages, scale in ((cache.k_pages.view(torch.uint8), cache.k_scale), (cache.v_pages.view(torch.uint8), cache.v_scale)):
                pages[b] = pages[a]
                scale[b] = scale[a]


def check(got, lse, want, out_dtype):
    """As for attend; joins multiply each part's sums by factors that are off by 2^-21, and add them up."""
    y, wl, a, top = want
    check_attend(got, lse, (y, wl, a + 2.0, top), out_dtype)


def ints(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


CASES = [
    # d, H, G, page, first places of groups, prefixes, held, new (None: one token each)
    (128, 2, 4, 16, [0, 4], [64], [64, 70, 100, 64], None),                        # 16 rows
    (128, 2, 4, 64, [0, 20], [192], [192 + 3 * i for i in range(20)], None),       # 80 rows: tcgen05
    (64, 3, 2, 32, [0, 3, 3, 5], [128, 500, 96], [130, 200, 128, 96, 300], None),  # an empty group
    (64, 1, 7, 16, [1, 3, 6], [80, 160], [33, 90, 81, 161, 170, 160, 5], None),    # places of no group
    (128, 1, 1, 128, [0, 3], [256], [256, -1, 300], None),                         # an idle member
    (128, 1, 8, 16, [0, 3], [150], [150, 151, 400], None),                         # no multiple of 64
    (64, 2, 2, 16, [0, 4], [200], [250, 131, 240, 500], None),                     # a member that is shorter
    (64, 2, 2, 16, [0, 3], [100], [20, 10, 300], None),                            # nothing left to share
    (128, 2, 4, 64, [0, 1, 3], [128, 128], [140, 128, 129], None),                 # a group of one
    (128, 1, 40, 16, [0, 2], [64], [70, 65], None),                                # more than 64 rows of two tokens
    (64, 1, 70, 16, [0, 2], [64], [70, 65], None),                                 # more than 64 rows of one token
    (128, 2, 4, 64, [0, 4], [256], [256, 300, 400, 256], [5, 3, 1, 4]),
    (64, 2, 3, 32, [0, 6], [320], [320 + 9 * i for i in range(6)], [6, 1, 5, 4, 2, 6]),
    (128, 1, 4, 64, [0, 3], [192], [192, 200, 250], [40, 100, 1]),                 # long own parts: tcgen05
    (64, 2, 2, 64, [0, 2, 4], [128, 64], [128, 140, 64, 90], [150, 0, 33, 2]),     # a member without tokens
    (128, 1, 3, 16, [0, 2], [64], [64, 64], [90, 200]),
    (64, 1, 4, 16, [2, 4], [64], [0, 700, 64, 66], [70, 1, 2, 1]),                 # long ones of no group
    (128, 2, 2, 1024, [0, 3], [1024], [1024, 1500, 2000], None),
]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES)
def test_shared(dev, case, out_dtype):
    d, H, G, page, first, prefix, held, new = case
    counts = new or [1] * len(held)
    table, lens, starts, total = shared_tables(first, prefix, held, counts, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    same_prefix(cache, table, first, prefix, held, page)
    hide_rest(cache, table, held, counts, page)
    q = (torch.randn((sum(counts), H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    want = attend_reference(cache, table, held, counts, q, page)
    kw = dict(starts=None if new is None else starts, out_dtype=out_dtype, want_lse=True, groups=ints(first, dev),
              prefix=ints(prefix, dev))
    out, lse = cache.attend(table, lens, q, max_new=max(counts), **kw)
    check(out, lse, want, out_dtype)
    assert status()[0] == 0
    again, lse2 = cache.attend(table, lens, q, max_new=max(counts), **kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    for hint in (None, 1):
        check(*cache.attend(table, lens, q, max_new=hint, **kw), want, out_dtype)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,n,G,prefix", [(128, 30, 4, 6400), (64, 9, 16, 9984), (128, 5, 2, 8000), (64, 70, 4, 3008)])
def test_prefixes_cut_over_many_parts(dev, d, n, G, prefix, out_dtype):
    """Long prefixes: positions cut over all SMs, with few and many rows, beside own parts of all lengths."""
    H, page = 1, 64
    first, held = [0, n], [prefix + (i * 37) % 300 for i in range(n)]
    table, lens, _, total = shared_tables(first, [prefix], held, [1] * n, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    hide_rest(cache, table, held, [1] * n, page)
    q = (torch.randn((n, H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, out_dtype=out_dtype, want_lse=True, groups=ints(first, dev), prefix=ints([prefix], dev))
    some = [0, 1, n // 2, n - 1]
    want = attend_reference(cache, table[some], [held[i] for i in some], [1] * len(some), q[some], page)
    check(out[some], lse[some], want, out_dtype)
    plain, plse = cache.attend(table, lens, q, out_dtype=torch.float32, want_lse=True)
    w = 2.0 ** -6 if out_dtype == torch.bfloat16 else 2.0 ** -15
    assert (out.float() - plain).abs().max().item() <= w * plain.abs().max().item()
    assert status()[0] == 0


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_nan_and_scales_far_apart(dev, out_dtype):
    """A NaN value in the prefix reaches its column of all members, one of a sequence's own that
    sequence; parts whose values' scales lie 2^190 apart keep their weights."""
    H, G, page, d, prefix = 1, 3, 16, 64, 64
    first, held = [0, 2, 25], [70, 80] + [66 + i for i in range(23)]
    table, lens, _, total = shared_tables(first, [prefix, prefix], held, [1] * 25, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    hide_rest(cache, table, held, [1] * 25, page)
    for s in (0, 2):
        cache.v_pages.view(torch.uint8)[int(table[s, 1]), 0, 4, 5] = 127
        cache.v_scale[table[s, :4].long()] = 2.0 ** 95
    cache.v_scale[table[:, 4].long()] = 2.0 ** -95
    cache.v_pages.view(torch.uint8)[int(table[1, 4]), 0, 3, 9] = 255
    q = (torch.randn((25, G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, out_dtype=out_dtype, want_lse=True, groups=ints(first, dev),
                            prefix=ints([prefix] * 2, dev))
    nan = torch.isnan(out).cpu()
    want = torch.zeros_like(nan)
    want[:, :, 5] = True
    want[1, :, 9] = True
    assert torch.equal(nan, want)
    y, wl, a, top = attend_reference(cache, table, held, [1] * 25, q, page)
    ok = ~want.numpy()
    eps = 2.0 ** -21 * (a + 2) + 2.0 ** -20 + (2.0 ** -21 if out_dtype == torch.float32 else 2.0 ** -11)
    top = np.full(top.shape, 448 * 2.0 ** 95)                  # (NaN among the values)
    tol = 2 * eps[..., None] * top[..., None] + (2.0 ** -23 if out_dtype == torch.float32 else 2.0 ** -8) * np.abs(y)
    assert (np.abs(out.double().cpu().numpy() - y)[ok] <= tol[ok]).all()
    assert (np.abs(lse.double().cpu().numpy() - wl) <= 2 * (2.0 ** -21 * (a + 2) + 2.0 ** -20) + 2.0 ** -22 * np.abs(wl)).all()


def test_weights_stay_where_own_values_are_heavy(dev):
    """The prefix's values are zeros at the smallest scale, the own ones large: the weights still share."""
    H, G, page, d, prefix = 1, 4, 16, 128, 128
    first, held = [0, 20], [140 + i for i in range(20)]
    table, lens, _, total = shared_tables(first, [prefix], held, [1] * 20, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    hide_rest(cache, table, held, [1] * 20, page)
    shared = table[0, :8].long()
    cache.v_pages.view(torch.uint8)[shared] = 0
    cache.v_scale[shared] = 2.0 ** -96
    cache.v_scale[table[:, 8:10].long().clamp_min(0)] = 2.0 ** 99
    cache.v_scale[shared] = 2.0 ** -96
    q = (torch.randn((20, G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    out, lse = cache.attend(table, lens, q, want_lse=True, groups=ints(first, dev), prefix=ints([prefix], dev))
    check(out, lse, attend_reference(cache, table, held, [1] * 20, q, page), torch.float32)


def test_idle_and_nobodys_rows(dev):
    H, G, page, d = 2, 2, 16, 64
    first, prefix, held, counts = [0, 5], [64], [64, -1, 70, 64, -1], [2, 3, 1, 1, 1]
    table, lens, starts, total = shared_tables(first, prefix, held, counts, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    hide_rest(cache, table, held, counts, page)
    q = (torch.randn((12, H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16()
    q[2:5] = math.nan
    q[7:] = math.nan
    q = q.to(dev)
    out, lse = torch.full((12, H * G, d), 7.0, device=dev), torch.full((12, H * G), 7.0, device=dev)
    cache.attend(table, lens, q, starts=starts, out=out, lse=lse, groups=ints(first, dev), prefix=ints(prefix, dev))
    want = attend_reference(cache, table, held, counts, q[:8].nan_to_num(0.0), page)
    check(out[:8], lse[:8], want, torch.float32)
    assert (out[2:5] == 0).all() and (lse[2:5] == -math.inf).all() and (out[8:] == 7).all() and (lse[8:] == 7).all()
    assert status()[0] == 0


def test_rows_before_the_first_sequence_stay(dev):
    """Many rows a sequence (tcgen05, positions in parts) and few, behind rows that are nobody's."""
    H, G, page, d, skip = 1, 4, 64, 128, 70
    first, prefix, held, counts = [0, 3], [512], [512, 600, 700], [90, 3, 40]
    table, lens, starts, total = shared_tables(first, prefix, held, counts, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    hide_rest(cache, table, held, counts, page)
    n = skip + sum(counts)
    q = (torch.randn((n, H * G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    out, lse = torch.full((n, H * G, d), 7.0, device=dev), torch.full((n, H * G), 7.0, device=dev)
    cache.attend(table, lens, q, starts=starts + skip, out=out, lse=lse, groups=ints(first, dev), prefix=ints(prefix, dev))
    assert status()[0] == 0 and (out[:skip] == 7).all() and (lse[:skip] == 7).all()
    check(out[skip:], lse[skip:], attend_reference(cache, table, held, counts, q[skip:], page), torch.float32)


def test_bad_groups_and_tables(dev):
    H, G, page, d = 1, 2, 16, 64
    first, prefix, held = [0, 3, 5], [64, 64], [70, 64, 90, 66, 65]
    table, lens, starts, total = shared_tables(first, prefix, held, [1] * 5, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    q = (torch.randn((5, G, d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    good, _ = cache.attend(table, lens, q, groups=ints(first, dev), prefix=ints(prefix, dev))
    plain, _ = cache.attend(table, lens, q)
    for bad in ([0, 6, 5], [-1, 3, 5], [0, 4, 3], [2 ** 31 - 1, -2 ** 31, 4]):
        got, _ = cache.attend(table, lens, q, groups=ints(bad, dev), prefix=ints(prefix, dev))
        assert status()[0] == 6
        if bad[0] == -1:
            assert (got - plain).abs().max().item() <= 2.0 ** -15 * plain.abs().max().item()
    for p in ([-5, 0], [63, -2 ** 31]):                         # nothing is shared: no error
        got, _ = cache.attend(table, lens, q, groups=ints(first, dev), prefix=ints(p, dev))
        assert status()[0] == 0 and (got - plain).abs().max().item() <= 2.0 ** -15 * plain.abs().max().item()
    got, _ = cache.attend(table, lens, q, groups=ints(first, dev), prefix=ints([2 ** 31 - 1, 64], dev))
    assert status()[0] == 0 and torch.equal(got[3:], good[3:])   # (as many as its members have)
    worse = table.clone()
    worse[0, 1] = total + 7                                      # the page of a prefix
    got, _ = cache.attend(worse, lens, q, groups=ints(first, dev), prefix=ints(prefix, dev))
    assert status()[0] == 6 and torch.equal(got[3:], good[3:])
    worse = table.clone()
    worse[3, 4] = -1                                             # a page of a sequence's own
    got, _ = cache.attend(worse, lens, q, groups=ints(first, dev), prefix=ints(prefix, dev))
    assert status()[0] == 6 and torch.equal(got[[0, 1, 2, 4]], good[[0, 1, 2, 4]])
    for s in ([0, 9, 3, 4, 5, 5], [0, 2, 1, 9, 9, 5], [-3, 1, 2, 3, 4, 5]):
        cache.attend(table, lens, q, starts=ints(s, dev), groups=ints(first, dev), prefix=ints(prefix, dev))
        assert status()[0] == 6
    got, _ = cache.attend(table, lens, q, groups=ints(first, dev), prefix=ints(prefix, dev))
    assert status()[0] == 0 and torch.equal(got, good)


def test_capture_streams_and_other_calls_of_one_workspace(dev):
    H, G, page, d = 2, 4, 64, 128
    first, prefix, held = [0, 24], [1024], [1024 + 7 * i for i in range(24)]
    table, lens, starts, total = shared_tables(first, prefix, held, [1] * 24, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    hide_rest(cache, table, held, [1] * 24, page)
    g = torch.Generator().manual_seed(5)
    q = (torch.randn((24, H * G, d), generator=g) * 0.02).bfloat16().to(dev)
    groups, pre = ints(first, dev), ints(prefix, dev)
    want, wl = cache.attend(table, lens, q, want_lse=True, groups=groups, prefix=pre)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, gl = cache.attend(table, lens, q, want_lse=True, groups=groups, prefix=pre, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(gl, wl)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(table, lens, q, out=out, groups=groups, prefix=pre)
        cache.attend(table, lens, q, out_dtype=torch.bfloat16)
        cache.attend(table, lens, q, out=out, groups=groups, prefix=pre)
    graph.replay()
    assert torch.equal(out, want)
    q.copy_((torch.randn(q.shape, generator=g) * 0.02).bfloat16())
    lens -= 3
    pre.fill_(1000)                                              # fewer than the shortest member has
    graph.replay()
    again, _ = cache.attend(table, lens, q, groups=groups, prefix=pre)
    assert torch.equal(out, again)
    check(out, *(lambda y, wl, a, top: (cache.attend(table, lens, q, groups=groups, prefix=pre, want_lse=True)[1],
                                        (y, wl, a, top)))(*attend_reference(cache, table, [h - 3 for h in held], [1] * 24, q, page)),
          torch.float32)


def test_results_over_the_queries_and_strided_queries(dev):
    H, G, page, d = 2, 2, 32, 64
    first, prefix, held = [0, 3], [96], [96, 100, 130]
    table, lens, starts, total = shared_tables(first, prefix, held, [1] * 3, page, dev, seed=3)
    cache = make_cache(dev, total, H, d, page, seed=2)
    same_prefix(cache, table, first, prefix, held, page)
    wide = (torch.randn((3, 2, H * G, 2 * d), generator=torch.Generator().manual_seed(5)) * 0.02).bfloat16().to(dev)
    q = wide[:, 1, :, d:].contiguous()
    kw = dict(groups=ints(first, dev), prefix=ints(prefix, dev))
    want, _ = cache.attend(table, lens, q, out_dtype=torch.bfloat16, **kw)
    got, _ = cache.attend(table, lens, wide[:, 1, :, d:], out_dtype=torch.bfloat16, **kw)
    assert torch.equal(got, want)
    cache.attend(table, lens, q, out=q, **kw)
    assert torch.equal(q, want)
