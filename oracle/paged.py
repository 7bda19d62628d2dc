"""Paged 8-bit key/value cache in 64 bits, one token and one row at a time, from the definitions:
the position rotation, e4m3 rounding under a power-of-two scale for each block of 16 tokens, and
softmax attention over what the cache then holds."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
E_MIN = -96
LIMIT = 2.0 ** 108

# value of every e4m3 byte: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN
E4M3 = np.array([(-1.0 if c & 128 else 1.0) *
                 (math.nan if c & 127 == 127 else
                  (c & 7) * 2.0 ** -9 if (c >> 3 & 15) == 0 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                 for c in range(256)])
_POSITIVE = E4M3[:127]


def round_e4m3(x):
    """Byte of the nearest e4m3 value, ties to the even byte; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(a >= _POSITIVE[126], 126, c)
    return np.where(np.isfinite(x), c + 128 * np.signbit(x), 127).astype(np.uint8)


def exponent(amax):
    """Least e >= E_MIN with amax <= 448 * 2^e."""
    e = E_MIN
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def rotate(x, cos, sin, interleaved=False):
    """One row x [d] by one row of the tables, [rot / 2] each."""
    y = np.array(x, dtype=np.float64)
    half = len(cos)
    for j in range(half):
        i, k = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        a, b = float(x[i]), float(x[k])
        y[i] = a * float(cos[j]) - b * float(sin[j])
        y[k] = b * float(cos[j]) + a * float(sin[j])
    return y


def append_token(codes, scale, row, x):
    """Puts x [d] at `row` of one block: codes [16][d] bytes and the block's scale; returns the
    scale."""
    fine = np.isfinite(x) & (np.abs(np.where(np.isfinite(x), x, 0.0)) < LIMIT)
    need = 2.0 ** exponent(np.abs(x[fine]).max(initial=0.0))
    old = 0.0 if row == 0 else scale
    new = max(need, old)
    if row and new > old:
        codes[:row] = round_e4m3(E4M3[codes[:row]] * (old / new))
    codes[row] = round_e4m3(np.where(fine, x, np.nan) / new)
    return new


def append_tokens(codes, scale, row, xs):
    """Puts xs [n][d] at rows row .. of one block at once; returns the scale."""
    fine = np.isfinite(xs) & (np.abs(np.where(np.isfinite(xs), xs, 0.0)) < LIMIT)
    need = 2.0 ** exponent(np.abs(xs[fine]).max(initial=0.0))
    old = 0.0 if row == 0 else scale
    new = max(need, old)
    if row and new > old:
        codes[:row] = round_e4m3(E4M3[codes[:row]] * (old / new))
    codes[row:row + len(xs)] = round_e4m3(np.where(fine, xs, np.nan) / new)
    return new


def attend(q, k, v):
    """One query row [d] over k, v [t][d]: (softmax(q k / sqrt(d)) v, natural-log normaliser)."""
    if len(k) == 0:
        return np.zeros(len(q)), -math.inf
    x = np.asarray(k, np.float64) @ np.asarray(q, np.float64) / math.sqrt(len(q))
    top = x.max()
    p = np.exp(x - top)
    return p @ np.asarray(v, np.float64) / p.sum(), top + math.log(p.sum())


def weights(q, k, lse):
    """What one query row [d] with normaliser lse gives to k [t][d]: exp(q k / sqrt(d) - lse); nothing
    where lse is -inf."""
    if lse == -math.inf:
        return np.zeros(len(k))
    return np.exp(np.asarray(k, np.float64) @ np.asarray(q, np.float64) / math.sqrt(len(q)) - float(lse))


def kept(mass, keep, sinks, window):
    """Positions that stay, ascending, of those that mass [t] has: one head's, taken one at a time."""
    n = len(mass)
    if n <= keep:
        return list(range(n))
    stay = list(range(sinks)) + list(range(n - window, n))
    rest = list(range(sinks, n - window))
    for _ in range(keep - sinks - window):
        best = rest[0]
        for t in rest:                                   # strictly larger: the lower position among equals
            a, b = (-math.inf if math.isnan(mass[i]) else float(mass[i]) for i in (t, best))
            if a > b:
                best = t
        rest.remove(best)
        stay.append(best)
    return sorted(stay)


def store_block(codes, scales):
    """Bytes [n][d] (n <= 16) of one new block, and its scale, from codes [n][d] under scales [n]."""
    x = E4M3[codes] * np.asarray(scales, np.float64)[:, None]
    scale = 2.0 ** exponent(np.abs(x[np.isfinite(x)]).max(initial=0.0))
    return round_e4m3(x / scale), scale
