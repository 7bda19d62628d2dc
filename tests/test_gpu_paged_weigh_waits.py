"""Waits of the attention weights' tcgen05 kernel: a model of its barriers, whose roles' steps are taken in
every order, and batches in which the roles reach a tile at very different times."""
import os
import re
from types import SimpleNamespace

import pytest
import torch

from conftest import ROOT
from test_gpu_paged import dev, hide_rest, make_cache, status, tables  # noqa: F401
from test_gpu_paged_weigh import check, start_mass
from test_gpu_paged_weigh_rows import logits, normalisers, reference

SOFT = 2                                                # softmax warps of the model, one of each half


def programs(tiles, blocks, softmax_gives_back, slots):
    """What each role does in order: waits for a phase of a barrier, and arrivals (the pipe's follow what the
    MMA warp has issued).  slots: query rows come anew for each block, through so many; 0: they stay."""
    keys, mma, pipe, rows = [], [], [], []
    soft = [[] for _ in range(SOFT)]

    def issue(barrier):
        mma.append(("arrive", "issued", 0))
        pipe.append(("wait", "issued", len(pipe) // 2))
        pipe.append(("arrive", barrier, 0))

    step = 0
    for i in range(tiles):
        if i >= 2:
            keys.append(("wait", f"AEMPTY{i & 1}", i // 2 - 1))
        keys.append(("arrive", f"AFULL{i & 1}", 0))
        for r in [mma] + soft:
            r.append(("wait", f"AFULL{i & 1}", i // 2))
        if softmax_gives_back:
            for r in soft:
                r.append(("arrive", f"AEMPTY{i & 1}", 0))
        for _ in range(blocks):
            if slots:
                st, k = step % slots, step // slots
                if k:
                    rows.append(("wait", f"EMPTY{st}", k - 1))
                rows.append(("arrive", f"FULL{st}", 0))
                for r in [mma] + soft:
                    r.append(("wait", f"FULL{st}", k))
            for hh in range(SOFT):
                if step:
                    mma.append(("wait", f"PFULL{hh}", step - 1))
                issue(f"SFULL{hh}")
                soft[hh].append(("wait", f"SFULL{hh}", step))
                soft[hh].append(("arrive", f"PFULL{hh}", 0))
            if slots:
                issue(f"EMPTY{st}")
                for r in soft:
                    r.append(("arrive", f"EMPTY{st}", 0))
            step += 1
        issue(f"AEMPTY{i & 1}")
    return [keys, mma, pipe, rows] + soft


def lost_waits(roles, counts):
    """Waits that some order of the roles' steps loses (they never pass again) or passes too early."""
    before = []                                         # arrivals of a role's first steps at each barrier
    for r in roles:
        at, seen = [{}], {}
        for kind, b, _ in r:
            if kind == "arrive":
                seen = {**seen, b: seen.get(b, 0) + 1}
            at.append(seen)
        before.append(at)
    bad, start = set(), (0,) * len(roles)
    todo, known = [start], {start}
    while todo:
        pc = todo.pop()
        moved = False
        for k, r in enumerate(roles):
            if pc[k] == len(r):
                continue
            kind, b, phase = r[pc[k]]
            if kind == "wait":
                came = sum(at[p].get(b, 0) for at, p in zip(before, pc))
                done = came // counts(b)
                if b == "issued":
                    if came <= phase:
                        continue
                else:
                    if done >= phase + 2 or (done < phase and done % 2 != phase % 2):
                        bad.add((k, b, phase))
                    if done % 2 == phase % 2:           # the phase that is open has this parity
                        continue
            moved = True
            to = pc[:k] + (pc[k] + 1,) + pc[k + 1:]
            if to not in known:
                known.add(to)
                todo.append(to)
        if not moved and any(p < len(r) for p, r in zip(pc, roles)):
            bad.add("stuck")
    return bad


def counts(both):
    return lambda b: {"AEMPTY": 1 + SOFT if both else 1, "EMPTY": 1 + SOFT}.get(b.rstrip("01"), 1)


@pytest.mark.parametrize("slots", [0, 2])
@pytest.mark.parametrize("tiles, blocks", [(5, 1), (4, 2)])
def test_no_order_loses_a_phase(tiles, blocks, slots):
    assert lost_waits(programs(tiles, blocks, True, slots), counts(True)) == set()


def test_one_consumer_is_not_enough():
    """Operands that the MMA warp alone gives back: with one block a tile a softmax warp's wait is lost."""
    assert "stuck" in lost_waits(programs(5, 1, False, 0), counts(False))


def test_the_kernel_counts_both_consumers():
    with open(os.path.join(ROOT, "paper_2607_05061_gb300", "csrc", "kvpop_paged_weigh_tc.cu")) as f:
        text = f.read()
    assert re.search(r"mbar_init\(bar\(L::AEMPTY \+ i\), 1 \+ WT_SOFT\)", text)
    assert len(re.findall(r"mbar_arrive\(bar\(L::AEMPTY", text)) == 1 and len(re.findall(r"commit\(bar\(L::AEMPTY", text)) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_runs_of_few_rows_between_many(dev, d):  # noqa: F811
    """Sequences of 40 to 120 rows (one block a tile, more than six tiles a CTA) with runs of 1, 10 and 200
    others between them, of one token, none, or idle, which every role of the kernel walks over by itself."""
    H, G, page = 2, 4, 16
    sms = torch.cuda.get_device_properties(dev).multi_processor_count
    held, new, tiles, i = [], [], 0, 0
    while tiles < 7 * sms:
        held.append(2600 + 257 * (i % 6))
        new.append(10 + i * 7 % 21)
        tiles += H * -(-(held[-1] + new[-1]) // 256)
        for j in range((1, 10, 200)[i % 3]):
            held.append(-1 if j % 3 == 1 else 3 + j % 40)
            new.append(int(j % 5 != 4))
        i += 1
    need = sum(-(-(max(p, 0) + n) // page) for p, n in zip(held, new))
    table, lens, starts = tables(held, new, page, need, dev, seed=61)
    cache = make_cache(dev, need, H, d, page, seed=62)
    hide_rest(cache, table, held, new, page)
    here = SimpleNamespace(H=H, d=d, k_pages=cache.k_pages.cpu(), k_scale=cache.k_scale.cpu())
    q = (torch.randn((sum(new), H * G, d), generator=torch.Generator().manual_seed(63)) * 0.02).bfloat16()
    x = logits(here, table.cpu(), held, new, q, page)
    lse = normalisers(x, sum(new), H, G, held, new)
    mass = start_mass(table, H, page, held)
    want, tol = reference(x, lse, mass, H, G, held, new)
    args = (table, lens, q.to(dev), lse.to(dev))
    first = cache.weigh(*args, mass.to(dev), starts=starts, max_new=max(new))
    assert status()[0] == 0
    check(first, want, tol)
    for _ in range(20):
        got = cache.weigh(*args, mass.to(dev), starts=starts, max_new=max(new))
        assert torch.equal(got.nan_to_num(nan=-1.0), first.nan_to_num(nan=-1.0))
    assert status()[0] == 0
