"""Outputs of the paged calls that share memory with what the calls read."""
import ctypes

import pytest
import torch

from test_paged_arguments import append, attend, batch, kv, pool, rows  # noqa: F401

SIZE = 1 << 16
BUF = (ctypes.c_char * (SIZE + 256))()
AT = (ctypes.addressof(BUF) + 255) // 256 * 256


def meets(spans, lo, hi):
    return any(a < hi and lo < b for a, b in spans)


# (token stride, head stride) of q in elements, [3 tokens][4 heads][64] bf16: together, columns of wider
# rows, heads first, heads apart, shared by the tokens, backwards
LAYOUTS = [(256, 64), (1024, 64), (64, 512), (2048, 128), (0, 64), (-256, 64), (256, -64)]


@pytest.mark.parametrize("ts,hs", LAYOUTS)
def test_rotated_queries_over_the_queries_are_refused(kv, ts, hs):  # noqa: F811
    """Every place of q_out that shares a byte with q; the places that do not are for the GPU."""
    n, heads, d = 3, 4, 64
    base = AT + SIZE // 2
    spans = [(base + 2 * (i * ts + h * hs), base + 2 * (i * ts + h * hs + d)) for i in range(n) for h in range(heads)]
    free = AT + SIZE - 2 * n * 2 * d                    # k and v are at the end
    far = rows(kv, data_dev=free, token_stride=128, head_stride=64)
    seen = 0
    for out in range(base - 8192, base + 14000, 16):
        if meets(spans, out, out + 2 * n * heads * d):
            b = batch(kv, n_seq=n, n_tokens=n)
            assert append(kv, b=b, q=rows(kv, data_dev=base, token_stride=ts, head_stride=hs), k=far, v=far,
                          q_out=out) == 1
            seen += 1
    assert seen > 90


@pytest.mark.parametrize("which", ["k", "v"])
def test_rotated_queries_over_keys_or_values_are_refused(kv, which):  # noqa: F811
    far = rows(kv, data_dev=AT + 16384)
    a = dict(q=far, k=rows(kv, data_dev=AT + 32768), v=rows(kv, data_dev=AT + 32768))
    a[which] = rows(kv, data_dev=AT + 1024 - 16)
    assert append(kv, q_out=AT, **a) == 1


@pytest.mark.parametrize("ts,hs", LAYOUTS)
def test_attention_over_other_rows_of_the_queries_is_refused(kv, ts, hs):  # noqa: F811
    n, heads, d = 3, 4, 64
    base = AT + SIZE // 2
    spans = [(base + 2 * (i * ts + h * hs), base + 2 * (i * ts + h * hs + d)) for i in range(n) for h in range(heads)]
    for dtype, size in ((kv.KVPOP_F32, 4), (kv.KVPOP_BF16, 2)):
        for out in range(base - 8192, base + 14000, 16):
            same = size == 2 and out == base and (ts, hs) == (256, 64)
            if meets(spans, out, out + size * n * heads * d) and not same:
                assert attend(kv, b=batch(kv, n_seq=n, n_tokens=n),
                              q=rows(kv, data_dev=base, token_stride=ts, head_stride=hs), out=out, dtype=dtype) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 5, 70])
def test_attention_in_place_of_the_queries(cuda_device, new):
    from test_gpu_paged import make_cache, tables
    H, G, d, page, held = 2, 4, 128, 16, [700, 30, 2000]
    cache = make_cache(cuda_device, 190, H, d, page, seed=61)
    table, lens, starts = tables(held, [new] * 3, page, 190, cuda_device, seed=62)
    q = (torch.randn((3 * new, H * G, d), generator=torch.Generator().manual_seed(63)) * 0.02).bfloat16().cuda()
    a = dict(starts=starts, max_new=new, out_dtype=torch.bfloat16)
    want, _ = cache.attend(table, lens, q, **a)
    for _ in range(10):
        x = q.clone()
        cache.attend(table, lens, x, out=x, **a)
        assert torch.equal(x, want)


@pytest.mark.gpu
def test_rotated_queries_beside_the_queries(cuda_device):
    """q_out in the memory that q's rows leave free."""
    from paper_2607_05061_gb300.paged import PagedCache
    H, G, d = 2, 4, 64
    HQ = H * G
    for n in (1, 2):
        cache = PagedCache.empty(2, H, d, page=16)
        table = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1)
        lens = torch.zeros(n, dtype=torch.int32, device="cuda")
        row = torch.randn(n, HQ + 2 * H + n * HQ, d, device="cuda").bfloat16()
        q, k, v = row[:, :HQ], row[:, HQ:HQ + H], row[:, HQ + H:HQ + 2 * H]
        want = cache.append(table, lens, q, k, v)
        out = row[0, HQ + 2 * H:].view(n, HQ, d)
        got = cache.append(table, lens, q, k, v, q_out=out)
        assert got is out and torch.equal(out, want) and torch.equal(out, q)
        with pytest.raises(Exception):
            cache.append(table, lens, q, k, v, q_out=row[0, HQ + 2 * H - 1:][:n * HQ].view(n, HQ, d))
