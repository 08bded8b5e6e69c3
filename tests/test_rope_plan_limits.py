"""Plans whose frequencies a fraction of a turn does not hold: refused, and the ones just inside (no GPU)."""
import ctypes
import math

import numpy as np
import pytest

from paper_2605_31105_gb300 import binding as b
from tests import rope_ref as R
from tests.test_abi import lib  # noqa: F401  (builds the library if it is stale)


# frequencies that overflow fp64, that are whole numbers of turns in it, and the first ones past the limit of
# 1024 radians a position
@pytest.mark.parametrize("kw,factors", [
    (dict(scaling="linear", factor=1e-320), None), (dict(scaling="linear", factor=1e-310), None),
    (dict(scaling="linear", factor=1e-20), None), (dict(scaling="linear", factor=2.0 ** -10), None),
    (dict(scaling="ntk", factor=1e-300), None), (dict(scaling="ntk", factor=1e-300, rotary=4), None),
    (dict(scaling="ntk", factor=1e-9, rotary=4), None), (dict(scaling="bands", factor=1e-320), None),
    (dict(scaling="bands", factor=1e-30), None), (dict(scaling="yarn", factor=1e-320), None),
    (dict(scaling="yarn", factor=1e-300, original=3.0), None), (dict(rotary=4), [1e-310, 1.0]),
    (dict(rotary=4), [1.0, 1e-308]), (dict(rotary=4), [2.0 ** -10, 1.0]),
    (dict(rotary=4, scaling="linear", factor=2.0 ** -5), [2.0 ** -5, 1.0])])
def test_frequencies_without_a_fraction_are_refused(lib, kw, factors):  # noqa: F811
    p = b.rope_params(**kw)
    out = b.grkv_rope()
    ctypes.memset(ctypes.byref(out), 0x5A, ctypes.sizeof(out))
    before = bytes(out)
    fac = None if factors is None else (ctypes.c_double * len(factors))(*factors)
    assert b.load().grkv_rope_make(ctypes.byref(p), fac, ctypes.byref(out)) == b.GRKV_ERR_INVALID_ARG
    assert bytes(out) == before


# The bound of test_frequencies (tests/test_rope_abi.py), 2^-48 of a frequency, of the whole frequency here: what is
# kept of it is its fraction of a turn.
@pytest.mark.parametrize("kw,factors", [
    (dict(scaling="linear", factor=2.0 ** -9), None), (dict(scaling="linear", factor=1e300), None),
    (dict(scaling="ntk", factor=0.5), None), (dict(scaling="ntk", factor=1e-4, rotary=4), None),
    (dict(scaling="ntk", factor=1e300, rotary=4), None), (dict(scaling="bands", factor=0.01), None),
    (dict(scaling="yarn", factor=1e-2, original=4096.0), None), (dict(rotary=4), [2.0 ** -9.99, 1e300])])
def test_frequencies_inside_the_limit(lib, kw, factors):  # noqa: F811
    r = b.grkv_rope_make(b.rope_params(**kw), factors)
    n = kw.get("rotary", 128) // 2
    f, _ = R.freqs(**kw, factors=factors)
    got = np.array(r.turns[:n], np.float64) / 2.0 ** 64
    turns = f / (2 * math.pi)
    off = np.abs(got - turns % 1.0)
    assert (np.minimum(off, 1 - off) <= turns * 2.0 ** -48 + 2.0 ** -64).all()
    assert f.max() < 1024
