"""Pins of the 64-bit implementation of weights and eviction: what it has to give by definition."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as op


def test_a_rows_weights_are_its_softmax():
    r = np.random.default_rng(1)
    q, k = r.standard_normal(64), r.standard_normal((50, 64))
    _, lse = op.attend(q, k, k)
    w = op.weights(q, k, lse)
    want = torch.softmax(torch.from_numpy(k @ q / 8.0), 0).numpy()
    assert np.abs(w - want).max() <= 1e-14 and abs(w.sum() - 1) <= 1e-13
    assert (op.weights(q, k, -math.inf) == 0).all()


@pytest.mark.parametrize("keep,sinks,window", [(1, 0, 0), (5, 2, 1), (7, 0, 7), (9, 4, 0), (12, 3, 3), (13, 0, 0), (40, 4, 2)])
def test_kept_is_the_best_set(keep, sinks, window):
    """Protected positions stay; no position that went outweighs one that stayed; ties go to the lower."""
    r = np.random.default_rng(2)
    for levels in (3, 1000):
        m = r.integers(0, levels, 13).astype(np.float64)
        m[4] = math.nan
        at = op.kept(m.tolist(), keep, sinks, window)
        assert at == sorted(set(at)) and len(at) == min(keep, 13)
        if keep >= 13:
            continue
        assert set(range(sinks)) <= set(at) and set(range(13 - window, 13)) <= set(at)
        key = np.where(np.isnan(m), -math.inf, m)
        free = [t for t in at if sinks <= t < 13 - window]
        gone = [t for t in range(sinks, 13 - window) if t not in at]
        assert all(key[g] < key[f] or (key[g] == key[f] and g > f) for g in gone for f in free)


def test_a_stored_block_is_what_append_would_store():
    """Rows of one block under its scale, moved whole: as appending their values; under scales that
    differ, each value is within half a step of the new scale's smallest codes of what it was."""
    r = np.random.default_rng(3)
    x = r.standard_normal((16, 64)) * 5
    codes = np.zeros((16, 64), np.uint8)
    scale = op.append_tokens(codes, 0.0, 0, x)
    new, s = op.store_block(codes, [scale] * 16)
    assert s == scale and np.array_equal(new, codes)
    again = np.zeros((16, 64), np.uint8)
    assert op.append_tokens(again, 0.0, 0, op.E4M3[codes] * scale) == s and np.array_equal(again, codes)
    scales = 2.0 ** r.integers(-12, 13, 16)
    new, s = op.store_block(codes, scales)
    was, now = op.E4M3[codes] * scales[:, None], op.E4M3[new] * s
    assert np.abs(now - was).max() <= s * 2.0 ** -10
    assert np.abs(was).max() <= 448 * s and np.abs(was).max() > 448 * s / 2
    assert op.store_block(np.zeros((3, 64), np.uint8), [1.0] * 3)[1] == 2.0 ** op.E_MIN


def test_nan_stays_and_does_not_count():
    codes = np.full((2, 64), 127, np.uint8)
    codes[0, :5] = 56                                   # 1.0
    new, s = op.store_block(codes, [4.0, 2.0 ** 60])
    assert s == 2.0 ** op.exponent(4.0) and (new[1] == 127).all() and (op.E4M3[new[0, :5]] * s == 4.0).all()
