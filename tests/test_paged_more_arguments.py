"""What append at positions, weights and eviction refuse, on the host: the C ABI by its status, the
binding by ValueError."""
import ctypes

import pytest
import torch

from test_paged_arguments import BAD_BATCH, BAD_POOL, PTR, batch, batch_args, cache, kv, pool, rows  # noqa: F401

AXES = (ctypes.c_char * 32)()


def append_at(kv, p=None, b=None, q=None, k=None, v=None, **kw):
    a = dict(n_q_heads=4, dtype=kv.KVPOP_BF16, cos=PTR, sin=PTR, rot=64, max_pos=8, inter=0, at=PTR, n_axes=3,
             axes=ctypes.addressof(AXES), q_out=PTR + 2048)
    a.update(kw)
    ref = ctypes.byref
    return kv.kvpop_paged_append_at(
        ref(p or pool(kv)), ref(b or batch(kv)), ref(q or rows(kv)), a["n_q_heads"], ref(k or rows(kv)),
        ref(v or rows(kv)), a["dtype"], a["cos"], a["sin"], a["rot"], a["max_pos"], a["inter"], a["at"], a["n_axes"],
        a["axes"], a["q_out"], None)


def weigh(kv, p=None, b=None, q=None, **kw):
    a = dict(heads=4, lse=PTR, mass=PTR + 2048, positions=64, ws=PTR, nbytes=1 << 40)
    a.update(kw)
    return kv.kvpop_paged_weigh(ctypes.byref(p or pool(kv)), ctypes.byref(b or batch(kv)), ctypes.byref(q or rows(kv)),
                                a["heads"], a["lse"], a["mass"], a["positions"], a["ws"], a["nbytes"], None)


def evict(kv, p=None, b=None, **kw):
    a = dict(mass=PTR, positions=64, to=PTR, stride=2, pages=2, keep=32, sinks=4, window=8, kept=PTR + 1024, new=None,
             new_positions=0, lens=None)
    a.update(kw)
    return kv.kvpop_paged_evict(ctypes.byref(p or pool(kv)), ctypes.byref(b or batch(kv)), a["mass"], a["positions"],
                                a["to"], a["stride"], a["pages"], a["keep"], a["sinks"], a["window"], a["kept"],
                                a["new"], a["new_positions"], a["lens"], None)


@pytest.mark.parametrize("bad", BAD_POOL)
def test_pools_that_are_refused(kv, bad):
    assert append_at(kv, p=pool(kv, **bad)) == 1
    assert weigh(kv, p=pool(kv, **bad)) == 1
    assert evict(kv, p=pool(kv, **bad)) == 1


@pytest.mark.parametrize("bad", BAD_BATCH)
def test_batches_that_are_refused(kv, bad):
    assert append_at(kv, b=batch(kv, **bad)) == 1
    assert weigh(kv, b=batch(kv, **bad)) == 1


@pytest.mark.parametrize("bad", [dict(n_seq=-1), dict(max_pages=0), dict(table_stride=3), dict(table_dev=None),
                                 dict(lens_dev=None)])
def test_batches_that_eviction_refuses(kv, bad):
    assert evict(kv, b=batch(kv, **bad)) == 1


@pytest.mark.parametrize("kw", [dict(at=None), dict(n_axes=0), dict(n_axes=5), dict(rot=0), dict(cos=None),
                                dict(max_pos=0), dict(q_out=None), dict(q_out=PTR), dict(at=PTR + 2048 + 1016)])
def test_append_at_arguments_that_are_refused(kv, kw):
    assert append_at(kv, **kw) == 1


def test_axes_that_are_none(kv):
    axes = (ctypes.c_uint8 * 32)(*([0] * 31 + [2]))
    assert append_at(kv, axes=ctypes.addressof(axes), n_axes=2) == 1
    axes[31] = 255
    assert append_at(kv, axes=ctypes.addressof(axes)) == 1


@pytest.mark.parametrize("kw", [dict(heads=0), dict(heads=3), dict(lse=None), dict(mass=None), dict(positions=63),
                                dict(positions=-1), dict(positions=1 << 60), dict(mass=PTR), dict(lse=PTR + 2048),
                                dict(ws=None)])
def test_weigh_arguments_that_are_refused(kv, kw):
    assert weigh(kv, **kw) == 1


def test_weigh_of_more_rows_than_an_int_numbers(kv):
    assert weigh(kv, b=batch(kv, starts_dev=PTR, n_tokens=2 ** 30)) == 1


@pytest.mark.parametrize("kw", [dict(mass=None), dict(positions=63), dict(to=None), dict(pages=0), dict(stride=1),
                                dict(keep=0), dict(keep=33), dict(sinks=-1), dict(window=-1), dict(sinks=20, window=13),
                                dict(kept=None), dict(kept=PTR + 512), dict(new=PTR + 512, new_positions=32),
                                dict(new=PTR + 1024, new_positions=32), dict(new=PTR + 2048, new_positions=31),
                                dict(lens=PTR + 4), dict(lens=PTR + 1028),
                                dict(lens=PTR + 252), dict(new=PTR + 8192, new_positions=32, lens=PTR + 8196), dict(sinks=2 ** 31 - 1, window=2 ** 31 - 1)])
def test_evict_arguments_that_are_refused(kv, kw):
    assert evict(kv, **kw) == 1


def test_eviction_of_more_than_a_grid_numbers(kv):
    assert evict(kv, b=batch(kv, n_seq=2 ** 27 + 1), p=pool(kv, n_kv_heads=2)) == 1
    assert evict(kv, b=batch(kv, n_seq=2 ** 26), p=pool(kv, n_kv_heads=2), keep=2 ** 13, pages=2 ** 9, stride=2 ** 9) == 1


def test_misaligned(kv):
    assert append_at(kv, at=PTR + 2) == 2 and append_at(kv, cos=PTR + 4) == 2 and append_at(kv, q_out=PTR + 2056) == 2
    assert weigh(kv, ws=PTR + 64) == 2
    assert weigh(kv, lse=PTR + 2) == 2 and weigh(kv, mass=PTR + 2050) == 2
    assert weigh(kv, q=rows(kv, data_dev=PTR + 2)) == 2 and weigh(kv, p=pool(kv, k_pages_dev=PTR + 8)) == 2
    assert evict(kv, kept=PTR + 1026) == 2 and evict(kv, to=PTR + 2) == 2 and evict(kv, lens=PTR + 3074) == 2
    assert evict(kv, new=PTR + 2050, new_positions=32) == 2 and evict(kv, p=pool(kv, v_pages_dev=PTR + 8)) == 2


def test_nothing_to_do_is_no_error(kv):
    empty = batch(kv, n_seq=0, n_tokens=0)
    assert append_at(kv, b=empty) == 0 and weigh(kv, b=empty) == 0 and evict(kv, b=empty) == 0
    none = batch(kv, starts_dev=PTR, n_tokens=0)
    assert append_at(kv, b=none) == 0 and weigh(kv, b=none) == 0


# ------------------------------------------------------------------ the binding
@pytest.mark.parametrize("what", ["axes alone", "no tables", "type", "rows", "three dimensions", "five axes",
                                  "no axis", "strided", "axes missing", "axes short", "axis 2", "axes for one", "device"])
def test_append_refuses_positions(cache, what):  # noqa: F811
    table, lens = batch_args()
    bf = torch.bfloat16
    at = torch.zeros(3, 2, dtype=torch.int32)
    a = dict(table=table, lens=lens, q=torch.zeros(3, 4, 64, dtype=bf), k=torch.zeros(3, 2, 64, dtype=bf),
             v=torch.zeros(3, 2, 64, dtype=bf), cos=torch.zeros(9, 32), sin=torch.zeros(9, 32), positions=at,
             axes=[0, 1] * 16)
    a.update({"axes alone": dict(positions=None), "no tables": dict(cos=None, sin=None), "type": dict(positions=at.long()),
              "rows": dict(positions=at[:2]), "three dimensions": dict(positions=at[None]),
              "five axes": dict(positions=torch.zeros(3, 5, dtype=torch.int32)),
              "no axis": dict(positions=torch.zeros(3, 0, dtype=torch.int32)),
              "strided": dict(positions=torch.zeros(2, 3, dtype=torch.int32).T), "axes missing": dict(axes=None),
              "axes short": dict(axes=[0, 1] * 15), "axis 2": dict(axes=[0, 2] * 16),
              "axes for one": dict(positions=torch.zeros(3, dtype=torch.int32)), "device": {}}[what])
    with pytest.raises(ValueError):
        cache.append(**a)


@pytest.mark.parametrize("what", ["q type", "heads", "lse type", "lse shape", "mass type", "mass heads", "mass short",
                                  "mass strided", "mass rows", "starts missing", "device"])
def test_weigh_refuses(cache, what):  # noqa: F811
    table, lens = batch_args()
    a = dict(table=table, lens=lens, q=torch.zeros(3, 4, 64, dtype=torch.bfloat16), lse=torch.zeros(3, 4),
             mass=torch.zeros(3, 2, 32))
    a.update({"q type": dict(q=a["q"].float()), "heads": dict(q=torch.zeros(3, 3, 64, dtype=torch.bfloat16)),
              "lse type": dict(lse=a["lse"].double()), "lse shape": dict(lse=torch.zeros(3, 2)),
              "mass type": dict(mass=a["mass"].half()), "mass heads": dict(mass=torch.zeros(3, 4, 32)),
              "mass short": dict(mass=torch.zeros(3, 2, 31)), "mass strided": dict(mass=torch.zeros(3, 2, 64)[..., ::2]),
              "mass rows": dict(mass=torch.zeros(4, 2, 32)),
              "starts missing": dict(q=torch.zeros(4, 4, 64, dtype=torch.bfloat16), lse=torch.zeros(4, 4)),
              "device": {}}[what])
    with pytest.raises(ValueError):
        cache.weigh(**a)


@pytest.mark.parametrize("what", ["to type", "to rows", "to strided", "keep none", "keep many", "sinks", "window",
                                  "protected", "mass short", "kept type", "kept shape", "new_mass short", "new_lens type",
                                  "lens type", "device"])
def test_evict_refuses(cache, what):  # noqa: F811
    table, lens = batch_args()
    a = dict(table=table, lens=lens, mass=torch.zeros(3, 2, 32), to=torch.zeros(3, 1, dtype=torch.int32), keep=16)
    a.update({"to type": dict(to=a["to"].long()), "to rows": dict(to=a["to"][:2]),
              "to strided": dict(to=torch.zeros(3, 2, dtype=torch.int32)[:, ::2].expand(3, 2)[:, :0]),
              "keep none": dict(keep=0), "keep many": dict(keep=17), "sinks": dict(sinks=-1), "window": dict(window=-1),
              "protected": dict(sinks=9, window=8), "mass short": dict(mass=torch.zeros(3, 2, 31)),
              "kept type": dict(kept=torch.zeros(3, 2, 16)), "kept shape": dict(kept=torch.zeros(3, 2, 15, dtype=torch.int32)),
              "new_mass short": dict(new_mass=torch.zeros(3, 2, 15)), "new_lens type": dict(new_lens=torch.zeros(3)),
              "lens type": dict(lens=lens.long()), "device": {}}[what])
    with pytest.raises(ValueError):
        cache.evict(**a)


# ------------------------------------------------------------------ shared prefixes
def shared(kv, p=None, b=None, q=None, **kw):
    a = dict(heads=4, groups=PTR, prefix=PTR, n=1, out=PTR + 2048, dtype=kv.KVPOP_F32, lse=PTR, ws=PTR, nbytes=1 << 40,
             scratch=PTR, sbytes=1 << 40)
    a.update(kw)
    return kv.kvpop_paged_attend_shared(
        ctypes.byref(p or pool(kv)), ctypes.byref(b or batch(kv)), ctypes.byref(q or rows(kv)), a["heads"], a["groups"],
        a["prefix"], a["n"], a["out"], a["dtype"], a["lse"], a["ws"], a["nbytes"], a["scratch"], a["sbytes"], None)


@pytest.mark.parametrize("bad", BAD_POOL)
def test_pools_that_shared_attention_refuses(kv, bad):
    assert shared(kv, p=pool(kv, **bad)) == 1


@pytest.mark.parametrize("bad", BAD_BATCH)
def test_batches_that_shared_attention_refuses(kv, bad):
    assert shared(kv, b=batch(kv, **bad)) == 1


@pytest.mark.parametrize("kw", [dict(heads=0), dict(heads=3), dict(groups=None), dict(prefix=None), dict(n=0), dict(n=-1),
                                dict(n=2 ** 30), dict(out=None), dict(dtype=5), dict(ws=None), dict(scratch=None),
                                dict(out=PTR)])
def test_shared_arguments_that_are_refused(kv, kw):
    assert shared(kv, **kw) == 1


def test_shared_alignment_and_nothing_to_do(kv):
    assert shared(kv, groups=PTR + 2) == 2 and shared(kv, prefix=PTR + 1) == 2 and shared(kv, scratch=PTR + 16) == 2
    assert shared(kv, b=batch(kv, n_seq=0, n_tokens=0)) == 0
    assert shared(kv, b=batch(kv, starts_dev=PTR, n_tokens=0)) == 0


def test_shared_bytes(kv):
    def need(n=1, heads=4, **kw):
        return kv.kvpop_paged_shared_bytes(ctypes.byref(pool(kv)), ctypes.byref(batch(kv, **kw)), n, heads)
    assert need() >= 2 * 4 * 2 * (64 + 2) * 4
    assert need(n=0) == 0 and need(heads=3) == 0 and need(n_seq=-1) == 0
    assert need(starts_dev=PTR, n_tokens=1000) > need(starts_dev=PTR, n_tokens=10)


@pytest.mark.parametrize("what", ["groups alone", "prefix alone", "groups type", "prefix type", "groups shape",
                                  "no groups", "device"])
def test_attend_refuses_groups(cache, what):  # noqa: F811
    table, lens = batch_args()
    i32 = torch.int32
    a = dict(table=table, lens=lens, q=torch.zeros(3, 4, 64, dtype=torch.bfloat16), groups=torch.zeros(2, dtype=i32),
             prefix=torch.zeros(1, dtype=i32))
    a.update({"groups alone": dict(prefix=None), "prefix alone": dict(groups=None), "groups type": dict(groups=torch.zeros(2)),
              "prefix type": dict(prefix=torch.zeros(1, dtype=torch.int64)), "groups shape": dict(groups=torch.zeros(3, dtype=i32)),
              "no groups": dict(groups=torch.zeros(1, dtype=i32), prefix=torch.zeros(0, dtype=i32)), "device": {}}[what])
    with pytest.raises(ValueError):
        cache.attend(**a)
