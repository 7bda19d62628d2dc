"""What the paged cache refuses, on the host: the C ABI by its status, the binding by ValueError,
and the page table's bookkeeping."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def kv():
    from paper_2607_05061_gb300 import build
    build.build()
    from paper_2607_05061_gb300 import kvpop
    return kvpop


BUF = (ctypes.c_char * 4096)()
PTR = (ctypes.addressof(BUF) + 255) // 256 * 256


def pool(kv, **kw):
    a = dict(k_pages_dev=PTR, v_pages_dev=PTR, k_scale_dev=PTR, v_scale_dev=PTR, n_pages=4, n_kv_heads=2,
             head_dim=64, page=16)
    a.update(kw)
    return kv.kvpop_paged_pool(**a)


def batch(kv, **kw):
    a = dict(table_dev=PTR, lens_dev=PTR, starts_dev=None, table_stride=4, max_pages=4, n_seq=2, n_tokens=2,
             max_new=1)
    a.update(kw)
    return kv.kvpop_paged_batch(**a)


def rows(kv, **kw):
    a = dict(data_dev=PTR, token_stride=128, head_stride=64)
    a.update(kw)
    return kv.kvpop_rows(**a)


def append(kv, p=None, b=None, q=None, k=None, v=None, **kw):
    a = dict(n_q_heads=4, dtype=kv.KVPOP_BF16, cos=PTR, sin=PTR, rot=64, max_pos=8, inter=0, q_out=PTR)
    a.update(kw)
    ref = ctypes.byref
    return kv.kvpop_paged_append(
        ref(p or pool(kv)), ref(b or batch(kv)), ref(q or rows(kv)), a["n_q_heads"], ref(k or rows(kv)),
        ref(v or rows(kv)), a["dtype"], a["cos"], a["sin"], a["rot"], a["max_pos"], a["inter"], a["q_out"], None)


def attend(kv, p=None, b=None, q=None, **kw):
    a = dict(heads=4, out=PTR, dtype=kv.KVPOP_F32, lse=PTR, ws=PTR, nbytes=1 << 40)
    a.update(kw)
    return kv.kvpop_paged_attend(ctypes.byref(p or pool(kv)), ctypes.byref(b or batch(kv)),
                                 ctypes.byref(q or rows(kv)), a["heads"], a["out"], a["dtype"], a["lse"], a["ws"],
                                 a["nbytes"], None)


BAD_POOL = [dict(k_pages_dev=None), dict(v_scale_dev=None), dict(n_pages=0), dict(n_kv_heads=0), dict(head_dim=96),
            dict(head_dim=256), dict(page=8), dict(page=48), dict(page=2048)]
BAD_BATCH = [dict(n_seq=-1), dict(n_tokens=-1), dict(n_tokens=3), dict(max_new=0), dict(max_pages=0),
             dict(table_stride=3), dict(table_dev=None), dict(lens_dev=None)]


@pytest.mark.parametrize("bad", BAD_POOL)
def test_pools_that_are_refused(kv, bad):
    assert append(kv, p=pool(kv, **bad)) == 1
    assert attend(kv, p=pool(kv, **bad)) == 1


@pytest.mark.parametrize("bad", BAD_BATCH)
def test_batches_that_are_refused(kv, bad):
    assert append(kv, b=batch(kv, **bad)) == 1
    assert attend(kv, b=batch(kv, **bad)) == 1


@pytest.mark.parametrize("kw", [dict(n_q_heads=0), dict(dtype=7), dict(cos=None), dict(rot=-16), dict(rot=24),
                                dict(rot=80), dict(max_pos=0), dict(inter=2), dict(q_out=None)])
def test_append_arguments_that_are_refused(kv, kw):
    assert append(kv, **kw) == 1


@pytest.mark.parametrize("kw", [dict(heads=0), dict(heads=3), dict(out=None), dict(dtype=5), dict(ws=None)])
def test_attend_arguments_that_are_refused(kv, kw):
    assert attend(kv, **kw) == 1


def test_more_heads_and_blocks_than_can_be_counted(kv):
    b = batch(kv, starts_dev=PTR, n_tokens=2 ** 31 - 1)
    assert append(kv, p=pool(kv, n_kv_heads=1 << 16), b=b) == 1


@pytest.mark.parametrize("name", ["k_pages_dev", "v_pages_dev"])
def test_misaligned_pages(kv, name):
    assert append(kv, p=pool(kv, **{name: PTR + 8})) == 2
    assert attend(kv, p=pool(kv, **{name: PTR + 8})) == 2


@pytest.mark.parametrize("kw", [dict(data_dev=PTR + 2), dict(token_stride=132), dict(head_stride=68)])
def test_misaligned_rows(kv, kw):
    assert append(kv, k=rows(kv, **kw)) == 2
    assert append(kv, q=rows(kv, **kw)) == 2
    assert attend(kv, q=rows(kv, **kw)) == 2


def test_misaligned_others(kv):
    assert append(kv, cos=PTR + 4) == 2
    assert append(kv, q_out=PTR + 8) == 2
    assert append(kv, b=batch(kv, lens_dev=PTR + 2)) == 2
    assert attend(kv, ws=PTR + 16) == 2
    assert attend(kv, out=PTR + 4) == 2
    assert attend(kv, lse=PTR + 2) == 2


def test_nothing_to_do_is_no_error(kv):
    empty = batch(kv, n_seq=0, n_tokens=0)
    assert append(kv, b=empty) == 0 and attend(kv, b=empty) == 0
    none = batch(kv, starts_dev=PTR, n_tokens=0)
    assert append(kv, b=none) == 0 and attend(kv, b=none) == 0


# ------------------------------------------------------------------ the binding
@pytest.fixture()
def cache(kv):
    from paper_2607_05061_gb300.paged import PagedCache
    return PagedCache.empty(4, 2, 64, page=16, device="cpu")


def batch_args():
    return torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)


def test_pages_of_other_types_and_shapes(kv):
    from paper_2607_05061_gb300.paged import PagedCache
    f8, u8 = torch.float8_e4m3fn, torch.uint8
    page = lambda *s: torch.zeros(s, dtype=u8).view(f8)  # noqa: E731
    s = torch.ones(4, 2, 1)
    PagedCache(page(4, 2, 16, 64), page(4, 2, 16, 64), s, s)
    for bad in ((page(4, 2, 16, 64).view(u8), page(4, 2, 16, 64), s, s),
                (page(4, 2, 16, 64), page(3, 2, 16, 64), s, s),
                (page(4, 2, 16, 64), page(4, 2, 16, 64), s[:, :1], s),
                (page(4, 2, 16, 64), page(4, 2, 16, 64), s, s.double()),
                (page(4, 16, 2, 64).transpose(1, 2), page(4, 2, 16, 64), s, s),
                (page(4, 2, 48, 64), page(4, 2, 48, 64), torch.ones(4, 2, 3), torch.ones(4, 2, 3)),
                (page(4, 2, 16, 32), page(4, 2, 16, 32), s, s)):
        with pytest.raises(ValueError):
            PagedCache(*bad)


@pytest.mark.parametrize("what", ["k dtype", "k heads", "k rows", "v dtype", "q width", "q inner", "table type",
                                  "table rows", "lens type", "starts", "starts missing", "cos alone", "cos width",
                                  "sin shape", "q_out alone", "q_out type", "device"])
def test_append_refuses(cache, what):
    table, lens = batch_args()
    bf = torch.bfloat16
    a = dict(table=table, lens=lens, q=torch.zeros(3, 4, 64, dtype=bf), k=torch.zeros(3, 2, 64, dtype=bf),
             v=torch.zeros(3, 2, 64, dtype=bf), cos=torch.zeros(9, 32), sin=torch.zeros(9, 32))
    a.update({"k dtype": dict(k=a["k"].half()), "k heads": dict(k=torch.zeros(3, 3, 64, dtype=bf)),
              "k rows": dict(k=torch.zeros(4, 2, 64, dtype=bf)), "v dtype": dict(v=a["v"].float()),
              "q width": dict(q=torch.zeros(3, 4, 32, dtype=bf)),
              "q inner": dict(q=torch.zeros(3, 64, 4, dtype=bf).transpose(1, 2)),
              "table type": dict(table=table.long()), "table rows": dict(table=table[:2]),
              "lens type": dict(lens=lens.float()), "starts": dict(starts=torch.zeros(3, dtype=torch.int32)),
              "starts missing": dict(k=torch.zeros(5, 2, 64, dtype=bf), v=torch.zeros(5, 2, 64, dtype=bf),
                                     q=torch.zeros(5, 4, 64, dtype=bf)),
              "cos alone": dict(sin=None), "cos width": dict(cos=torch.zeros(9, 20), sin=torch.zeros(9, 20)),
              "sin shape": dict(sin=torch.zeros(8, 32)), "q_out alone": dict(q=None, q_out=torch.zeros(3, 4, 64)),
              "q_out type": dict(q_out=torch.zeros(3, 4, 64)), "device": {}}[what])
    with pytest.raises(ValueError):
        cache.append(**a)


@pytest.mark.parametrize("what", ["q type", "heads", "out type", "out shape", "lse shape", "device"])
def test_attend_refuses(cache, what):
    table, lens = batch_args()
    a = dict(table=table, lens=lens, q=torch.zeros(3, 4, 64, dtype=torch.bfloat16))
    a.update({"q type": dict(q=a["q"].float()), "heads": dict(q=torch.zeros(3, 3, 64, dtype=torch.bfloat16)),
              "out type": dict(out=torch.zeros(3, 4, 64).half()), "out shape": dict(out=torch.zeros(3, 4, 32)),
              "lse shape": dict(lse=torch.zeros(3, 2)), "device": {}}[what])
    with pytest.raises(ValueError):
        cache.attend(**a)


def test_page_table(kv):
    from paper_2607_05061_gb300.paged import PageTable
    t = PageTable(3, 4, 6, page=16, device="cpu")
    assert t.lens.tolist() == [-1, -1, -1]
    t.open(0)
    t.open(2)
    t.grow([17, 5, 16])
    assert [len(p) for p in t.pages] == [2, 0, 1] and t.starts([17, 5, 16]).tolist() == [0, 17, 17, 33]
    t.advance([17, 5, 16])
    assert t.lens.tolist() == [17, -1, 16]
    t.grow(1)
    assert [len(p) for p in t.pages] == [2, 0, 2]
    t.advance(1)
    used = sorted(t.pages[0] + t.pages[2])
    assert len(set(used)) == 4 and all(t.dev[s, i] == p for s in (0, 2) for i, p in enumerate(t.pages[s]))
    with pytest.raises(MemoryError):
        t.grow([3 * 16, 0, 0])                     # a fifth page of one sequence
    t.open(1)
    before = [list(p) for p in t.pages]
    with pytest.raises(MemoryError):
        t.grow([0, 48, 0])                         # three pages, two are free
    assert t.pages == before
    t.close(0)
    assert t.lens.tolist() == [-1, 0, 18 - 1] and len(t.free) == 4 and t.dev[0].tolist() == [-1] * 4
    with pytest.raises(ValueError):
        t.grow([1, 1])
    with pytest.raises(ValueError):
        t.advance([-1, 0, 0])
