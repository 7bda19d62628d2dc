"""Pins of the paged cache's 64-bit oracle: e4m3 values and rounding against their definition and
torch's conversion, scales, rotation against complex products, attention against torch."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as op


def test_e4m3_values_match_torch():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(op.E4M3))
    fine = ~np.isnan(t)
    assert np.array_equal(t[fine], op.E4M3[fine])


def test_rounding_matches_torch_and_takes_ties_to_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000), op._POSITIVE,
                        (op._POSITIVE[1:] + op._POSITIVE[:-1]) / 2, [0.0, -0.0, 448.0, -448.0]])
    x = np.float32(np.clip(x, -448, 448)).astype(np.float64)
    want = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(op.round_e4m3(x), want)
    assert set(op.round_e4m3([math.inf, -math.inf, math.nan])) == {127}


@pytest.mark.parametrize("amax,e", [(0.0, -96), (448.0, 0), (448.1, 1), (1.0, -8), (0.875, -9), (0.876, -8),
                                    (2.0 ** 107, 99), (1e-30, -96)])
def test_scale_exponents(amax, e):
    assert op.exponent(amax) == e


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, ang = rng.normal(size=12), rng.normal(size=4)
    y = op.rotate(x, np.cos(ang), np.sin(ang), interleaved)
    z = (x[0:8:2] + 1j * x[1:8:2]) if interleaved else (x[:4] + 1j * x[4:8])
    z = z * np.exp(1j * ang)
    got = (y[0:8:2] + 1j * y[1:8:2]) if interleaved else (y[:4] + 1j * y[4:8])
    assert np.allclose(got, z, rtol=1e-15, atol=1e-15) and np.array_equal(y[8:], x[8:])


def test_tokens_one_by_one_and_at_once_agree_but_for_the_smallest_codes():
    rng = np.random.default_rng(2)
    xs = rng.normal(size=(16, 64)) * 2.0 ** rng.integers(-3, 6, (16, 1))
    a, b, sa = np.zeros((16, 64), np.uint8), np.zeros((16, 64), np.uint8), 0.0
    for i, x in enumerate(xs):
        sa = op.append_token(a, sa, i, x)
    assert sa == op.append_tokens(b, 0.0, 0, xs)
    va, vb = op.E4M3[a], op.E4M3[b]
    large = np.abs(vb) >= 2.0 ** -6
    # a code that stayed normal was only shifted: at most one step (2^-9) apart where it is not
    assert np.abs(va - vb)[~large].max(initial=0) <= 2.0 ** -9
    assert np.mean(va[large] == vb[large]) > 0.999


def test_attention_matches_torch():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=64), rng.normal(size=(37, 64)), rng.normal(size=(37, 64))
    y, lse = op.attend(q, k, v)
    t = torch.nn.functional.scaled_dot_product_attention(*(torch.tensor(x)[None, None] for x in (q[None], k, v)))
    assert np.allclose(y, t.numpy()[0, 0, 0], rtol=1e-12, atol=1e-12)
    assert abs(lse - np.log(np.exp(k @ q / 8).sum())) < 1e-12
    assert op.attend(q, k[:0], v[:0])[1] == -math.inf
