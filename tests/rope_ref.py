"""Plain forms of rotary positions in numpy and 64 bits, with the bounds of their arithmetic.

An angle is held to pi 2^-27 radians (a rest of at most an eighth of a turn in fp32) and 2^-32 turns
(the upper half of the 64-bit fraction) and its frequency to some 2^-51 of itself, so to
delta = 2^-25 + p f 2^-50.  Cosine and sine add 2^-23; times a (itself rounded) 2 x 2^-24; the two
products and their sum 2 x 2^-24 of |x| + |y|.  So an output is off by
  (delta + 2^-23 + 4 x 2^-24) a (|x| + |y|) + half a step of its type.
In bf16 the angle lies within half a turn, which fp32 rounds by pi 2^-24 twice (from 32 bits, and times
2 pi), and the special function unit's documented errors are 2^-21.41 and 2^-21.19: together 2^-20 in the
place of 2^-25 + 2^-23.
"""
import math

import numpy as np

from tests.cache_ref import D, ROUND

BIG = 2.0 ** -25 + 2.0 ** -23 + 4 * 2.0 ** -24
MORE_BF16 = 2.0 ** -20 - 2.0 ** -25 - 2.0 ** -23


def freqs(rotary=D, scaling="plain", theta=10000.0, factor=1.0, low=0.0, high=0.0, original=8192.0,
          amplitude=0.0, factors=None, layout=None):
    """Radians a position of every pair, and a."""
    low = low or 1.0
    high = high or (32.0 if scaling == "yarn" else 4.0)
    out = []
    for i in range(rotary // 2):
        f = math.exp(-2.0 * i / rotary * math.log(theta))
        if scaling == "linear":
            f = f / factor
        if scaling == "ntk" and rotary > 2:
            f = math.exp(-2.0 * i / rotary * (math.log(theta) + rotary / (rotary - 2) * math.log(factor)))
        if scaling == "bands":
            turns = original * f / (2 * math.pi)
            k = 0.0 if turns < low else 1.0 if turns > high else (turns - low) / (high - low)
            f = k * f + (1 - k) * f / factor
        if scaling == "yarn":
            dim = lambda t: rotary * math.log(original / (2 * math.pi * t)) / (2 * math.log(theta))
            a, b = max(math.floor(dim(high)), 0), min(math.ceil(dim(low)), rotary - 1)
            ramp = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            f = f / factor * ramp + f * (1 - ramp)
        if factors is not None:
            f = f / factors[i]
        out.append(f)
    a = amplitude or (0.1 * math.log(factor) + 1 if scaling == "yarn" and factor > 1 else 1.0)
    return np.array(out), a


def pairs(rotary, layout):
    i = np.arange(rotary // 2)
    return (i, i + rotary // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rotate(x, pos, layout="half", transpose=False, amplitude=None, dtype="f32", **kw):
    """x [..., D] float64 at positions pos [...] -> rotated, and a bound of the error before the
    output's own rounding."""
    f, a = freqs(**kw)
    a = a if amplitude is None else amplitude
    p = np.asarray(pos, np.float64)[..., None]
    ang = p * f * (-1 if transpose else 1)
    i, j = pairs(2 * len(f), layout)
    out, err = np.array(x, np.float64), np.zeros(np.shape(x))
    with np.errstate(invalid="ignore"):
        u, v = x[..., i], x[..., j]
        out[..., i] = a * (u * np.cos(ang) - v * np.sin(ang))
        out[..., j] = a * (u * np.sin(ang) + v * np.cos(ang))
        both = a * (np.abs(u) + np.abs(v))
        e = (BIG + np.abs(p * f) * 2.0 ** -50) * both
        if dtype == "bf16":
            e = e + MORE_BF16 * both
    err[..., i] = err[..., j] = e
    return out, err


def check(got, want, err, dtype):
    """got within err and half a step of want; NaN and infinities are not looked at here."""
    tol = err + ROUND[dtype] * (np.abs(want) + err)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want).max()), np.argwhere(bad)[:4].tolist())
