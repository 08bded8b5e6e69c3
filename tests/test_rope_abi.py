"""Rotary positions, positions and slots, attention over encoder states: plans and refusals (no
GPU: they are made before any CUDA call)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import rope_ref as R
from tests.test_abi import lib  # noqa: F401  (builds the library if it is stale)

FAKE = 1 << 20   # never dereferenced: every check below fails on the host


def test_defaults(lib):  # noqa: F811
    p = b.rope_params()
    assert (p.d, p.rotary, p.layout, p.scaling) == (128, 128, b.GRKV_ROPE_HALF, b.GRKV_ROPE_PLAIN)
    assert (p.theta, p.factor, p.low, p.high, p.original, p.amplitude) == (10000, 1, 0, 0, 8192, 0)


# A frequency goes through a power, a logarithm's rounding in the other side's formula, a product and
# a quotient by 2 pi: some 2^-50 of itself at the smallest (an exponent of 12 carries the rounding of
# a logarithm 12-fold: 12 x 2^-53), and half a unit of 2^-64 turns.
@pytest.mark.parametrize("rotary", [2, 4, 50, 64, 128])
@pytest.mark.parametrize("kw", [
    dict(), dict(theta=500000.0), dict(scaling="linear", factor=4.0), dict(scaling="linear", factor=0.25),
    dict(scaling="ntk", factor=8.0), dict(scaling="bands", factor=8.0),
    dict(scaling="bands", factor=32.0, theta=500000.0, low=0.5, high=9.0, original=2048.0),
    dict(scaling="yarn", factor=16.0, original=4096.0), dict(scaling="yarn", factor=2.5, low=2.0, high=8.0),
    dict(scaling="yarn", factor=4.0, original=3.0), dict(amplitude=0.75),
    dict(scaling="yarn", factor=4.0, amplitude=1.25), dict(scaling="yarn", factor=0.5)])
def test_frequencies(lib, rotary, kw):  # noqa: F811
    r = b.grkv_rope_make(b.rope_params(rotary=rotary, **kw))
    f, a = R.freqs(rotary, **kw)
    assert (r.rotary, r.layout) == (rotary, 0) and abs(r.amplitude / a - 1) < 2.0 ** -23
    got = np.array([x for x in r.turns[:rotary // 2]], np.float64) / 2.0 ** 64
    want = f / (2 * math.pi) % 1.0
    assert (np.abs(got - want) <= want * 2.0 ** -48 + 2.0 ** -64).all()
    assert not any(r.turns[rotary // 2:])


def test_free_factors(lib):  # noqa: F811
    fac = [1.0 + 0.5 * i for i in range(32)]
    r = b.grkv_rope_make(b.rope_params(rotary=64, layout="pairs"), fac)
    f, _ = R.freqs(64, factors=fac)
    got = np.array(r.turns[:32], np.float64) / 2.0 ** 64
    # as above: a 64-bit fraction cannot hold 1.3e-6 to 2^-48 of itself, half its unit is 2^-45.4 of that
    assert r.layout == b.GRKV_ROPE_PAIRS and np.allclose(got, f / (2 * math.pi), rtol=2.0 ** -48, atol=2.0 ** -64)
    with pytest.raises(ValueError, match="31 factors"):
        b.grkv_rope_make(b.rope_params(rotary=64), fac[:31])
    for bad in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(b.GrkvError):
            b.grkv_rope_make(b.rope_params(rotary=64), fac[:31] + [bad])


@pytest.mark.parametrize("kw,code", [
    (dict(rotary=0), -1), (dict(rotary=3), -1), (dict(rotary=130), -1), (dict(rotary=-2), -1),
    (dict(layout=2), -1), (dict(scaling=5), -1), (dict(scaling=-1), -1), (dict(theta=1.0), -1),
    (dict(theta=math.nan), -1), (dict(theta=math.inf), -1), (dict(scaling="linear", factor=0.0), -1),
    (dict(scaling="ntk", factor=math.inf), -1), (dict(scaling="yarn", factor=2.0, original=0.0), -1),
    (dict(scaling="bands", factor=2.0, low=4.0, high=4.0), -1),
    (dict(scaling="bands", factor=2.0, low=-1.0), -1), (dict(scaling="bands", factor=2.0, low=5.0), -1),
    (dict(scaling="yarn", factor=2.0, high=math.inf), -1), (dict(amplitude=-1.0), -1),
    (dict(amplitude=math.inf), -1), (dict(amplitude=1e300), -1), (dict(d=0), -1), (dict(d=64, rotary=64), -2),
    (dict(d=256), -2)])
def test_plans_that_are_refused(lib, kw, code):  # noqa: F811
    with pytest.raises(b.GrkvError) as e:
        b.grkv_rope_make(b.rope_params(**kw))
    assert e.value.code == code
    assert b.load().grkv_rope_make(None, None, ctypes.byref(b.grkv_rope())) == -1
    assert b.load().grkv_rope_make(ctypes.byref(b.rope_params()), None, None) == -1


def plan(**kw):
    r = b.grkv_rope_make(b.rope_params())
    for key, val in kw.items():
        setattr(r, key, val)
    return r


BAD_PLANS = [dict(rotary=0), dict(rotary=5), dict(rotary=130), dict(layout=2), dict(amplitude=0.0),
             dict(amplitude=math.nan), dict(amplitude=math.inf)]


def rows(seqs=2, heads=3, tokens=4, d=128, dtype=b.GRKV_BF16, flags=0, ins=(1536, 512, 128),
         outs=(1536, 512, 128), rope=None, x=FAKE, out=2 * FAKE, pos=None, start=None):
    r = b.grkv_rows(seqs, heads, tokens, d, dtype, flags, ins, outs)
    return b.load().grkv_rope_rows(rope or plan(), r, x, out, pos, start, None)


@pytest.mark.parametrize("kw,code", [
    (dict(seqs=-1), -1), (dict(heads=-1), -1), (dict(tokens=-1), -1), (dict(d=0), -1), (dict(d=64), -2),
    (dict(dtype=3), -1), (dict(flags=2), -1), (dict(pos=FAKE, start=FAKE), -1),
    (dict(seqs=1 << 16, tokens=(1 << 14) + 1), -2), (dict(heads=(1 << 16) + 1), -2),
    (dict(x=0), -1), (dict(out=0), -1), (dict(x=FAKE + 8), -4), (dict(out=FAKE + 2), -4),
    (dict(pos=FAKE + 2), -4), (dict(start=FAKE + 1), -4),
    (dict(ins=(1540, 512, 128)), -4), (dict(outs=(1536, 512, 132)), -4),
    (dict(ins=(1538, 512, 128), dtype=b.GRKV_F32), -4), (dict(ins=(-1536, 512, 128)), -1),
    (dict(outs=(1536, 512, 120)), -1), (dict(outs=(1536, 0, 128)), -1), (dict(outs=(128, 512, 128)), -1),
    (dict(outs=(1536, 384, 128)), -1), (dict(outs=(1408, 512, 128)), -1),
    (dict(out=FAKE, outs=(1536, 128, 384)), -1), (dict(out=FAKE, ins=(0, 512, 128)), -1),
    (dict(outs=(1536, (1 << 39) + 8, 128)), -1), (dict(ins=(1536, 1 << 40, 128)), -1)])
def test_rows_that_are_refused(lib, kw, code):  # noqa: F811
    assert rows(**kw) == code


@pytest.mark.parametrize("kw", BAD_PLANS)
def test_changed_plans_are_refused(lib, kw):  # noqa: F811
    p = b.cache_params(8, 4, 100, 64, 32)
    ws = dict(ws_bytes=b.grkv_cache_workspace_size(p), stream=0, check=False)
    assert rows(rope=plan(**kw)) == -1
    assert b.grkv_cache_append_rope(p, plan(**kw), *[FAKE] * 7, **ws) == -1
    assert b.grkv_cache_compact_rope(p, plan(**kw), *[FAKE] * 7, **ws) == -1


def test_no_rows_are_no_call(lib):  # noqa: F811
    for kw in (dict(seqs=0), dict(heads=0), dict(tokens=0)):
        assert rows(x=0, out=0, **kw) == b.GRKV_OK


def calls(p, ws_bytes, at=None, over=FAKE, ws=FAKE):
    """The cache calls with `over` as their pointer argument number `at`."""
    def f(n):
        args = [FAKE] * n
        if at is not None:
            args[at] = over
        return args
    kw = dict(ws_bytes=ws_bytes, stream=0, check=False)
    n = -1 if at is None else at
    return [fn(p, *lead, *f(m), ws, **kw) for fn, lead, m in (
        (b.grkv_attend_cross, (), 6), (b.grkv_cache_map, (), 4),
        (b.grkv_cache_append_rope, (plan(),), 6), (b.grkv_cache_compact_rope, (plan(),), 6)) if n < m]


def test_workspace_and_pointers(lib):  # noqa: F811
    p = b.cache_params(8, 4, 100, 64, 32)
    need = b.grkv_cache_workspace_size(p)
    assert calls(p, need - 1) == [b.GRKV_ERR_WORKSPACE_TOO_SMALL] * 4
    assert calls(p, need, ws=0) == [b.GRKV_ERR_INVALID_ARG] * 4
    assert calls(p, need, ws=FAKE + 8) == [b.GRKV_ERR_MISALIGNED] * 4
    for at in range(6):
        for over, code in ((0, b.GRKV_ERR_INVALID_ARG), (FAKE + 2, b.GRKV_ERR_MISALIGNED)):
            got = calls(p, need, at, over)
            assert got and got == [code] * len(got), (at, over)


def test_optional_arguments(lib):  # noqa: F811
    p = b.cache_params(8, 4, 100, 64, 32)
    kw = dict(ws_bytes=b.grkv_cache_workspace_size(p), stream=0, check=False)
    inv, mis = b.GRKV_ERR_INVALID_ARG, b.GRKV_ERR_MISALIGNED
    append = lambda **k: b.grkv_cache_append_rope(p, plan(), *[FAKE] * 7, **kw, **k)
    assert append(pos=FAKE, offset=FAKE) == inv
    assert append(q=FAKE) == inv and append(q_out=FAKE) == inv
    assert append(q=FAKE, q_out=FAKE + 4) == mis and append(q=FAKE + 8, q_out=FAKE) == mis
    for name in ("pos", "offset", "count"):
        assert append(**{name: FAKE + 2}) == mis
    assert append(first_row=FAKE + 4, new_rows=3) == mis and append(first_row=FAKE, new_rows=-1) == inv
    for name in ("keep", "first", "turn"):
        assert b.grkv_cache_compact_rope(p, plan(), *[FAKE] * 7, **kw, **{name: FAKE + 2}) == mis
    cross = lambda **k: b.grkv_attend_cross(p, *[FAKE] * 7, **kw, **k)
    assert cross(q_lens=FAKE + 2) == mis and cross(lse=FAKE + 2) == mis
    mapped = lambda q, **k: b.grkv_cache_map(q, *[FAKE] * 5, **dict(
        kw, ws_bytes=b.grkv_cache_workspace_size(q)), **k)
    for name, code in (("count", mis), ("parent", mis), ("offset", mis), ("first_row", mis)):
        assert mapped(p, **{name: FAKE + 2}) == code
    assert b.grkv_cache_map(p, FAKE, FAKE, FAKE, FAKE + 4, FAKE, **kw) == mis
    assert mapped(b.cache_params(8, 4, 100, 64, 32, tokens=257), parent=FAKE) == b.GRKV_ERR_UNSUPPORTED
    big = b.cache_params((1 << 20) + 1, 1, 100, 64, 1)
    assert mapped(big, first_row=FAKE) == b.GRKV_ERR_UNSUPPORTED
    q = b.cache_params(1, 1, 100, 128, 1 << 21, tokens=1 << 24, window=100)   # a window is not read
    assert b.grkv_attend_cross(q, *[FAKE] * 7, ws_bytes=b.grkv_cache_workspace_size(q), stream=0,
                               check=False) == b.GRKV_ERR_UNSUPPORTED


def test_tensors_are_checked_by_the_binding(lib):  # noqa: F811
    x = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16)
    for word, a, o in (("two .S, H, t, d", x[0], x[0]), ("two .S, H, t, d", x, x[:, :2]),
                       ("bfloat16 or float32", x.half(), x.half()), ("bfloat16 or float32", x, x.float()),
                       ("not contiguous", x.transpose(2, 3).contiguous().transpose(2, 3), x),
                       ("current CUDA device", x, x)):
        with pytest.raises(ValueError, match=word):
            b.grkv_rope_rows(plan(), a, o)
    p = b.cache_params(8, 4, 100, 64, 32)
    kw = dict(ws_bytes=b.grkv_cache_workspace_size(p), stream=0)
    i32, f = torch.zeros(8, 1, dtype=torch.int32), FAKE
    with pytest.raises(ValueError, match="pos is torch.int64"):
        b.grkv_cache_append_rope(p, plan(), *[f] * 7, pos=i32.long(), **kw)
    with pytest.raises(ValueError, match="q_out is torch.float32"):
        b.grkv_cache_append_rope(p, plan(), *[f] * 7, q=f, q_out=torch.zeros(8, 4, 1, 128, dtype=torch.float32), **kw)
    with pytest.raises(ValueError, match="turn is torch.int64"):
        b.grkv_cache_compact_rope(p, plan(), *[f] * 7, turn=i32.long(), **kw)
    with pytest.raises(ValueError, match="slot is torch.int32"):
        b.grkv_cache_map(p, f, f, f, i32, f, **kw)
    with pytest.raises(ValueError, match="first_row holds 8"):
        b.grkv_cache_map(p, f, f, f, f, f, first_row=torch.zeros(8, dtype=torch.int64), **kw)
    with pytest.raises(ValueError, match="new_rows"):
        b.grkv_cache_append_rope(p, plan(), *[f] * 7, first_row=f, **kw)
