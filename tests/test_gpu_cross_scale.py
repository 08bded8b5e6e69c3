"""grkv_attend_cross with scales near the end of fp32's range, whose products with queries and keys are ordinary."""
import math

import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R
from tests.test_gpu_attend import TYPES, queries
from tests.test_gpu_attend_cross import check, run

pytestmark = pytest.mark.gpu
ROWS = [(1, 1), (2, 1), (4, 1), (8, 1), (9, 1), (7, 30), (64, 2)]   # every kernel of fp32 and bf16


# Logits of ten at most: queries of 2^-100, keys of 2^-28.  The tolerance is cache_ref's, relative to scale |q| |k|:
# 130 x 2^-24 of it; what three bf16 parts lose below 2^-125 of a query of 2^-100 is 2^-25.
@pytest.mark.parametrize("dtype,flags", TYPES + [("f32", b.GRKV_FORCE_SIMT)])
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("scale", [2.0 ** 124, 2.0 ** 126, 1.25 * 2.0 ** 126, 2.0 ** 127])
def test_large_scales(grkv_lib, dtype, flags, g, t, scale):
    c = R.Cache([300, 65, 1, 0], 32, dtype, 70)
    c.k = c.k * 2.0 ** -28                       # powers of two: exact in either type
    q, q64 = queries(4, g, t, dtype, 71)
    q, q64 = q * 2.0 ** -100, q64 * 2.0 ** -100
    p = b.cache_params(4, g, c.pages, 32, c.cols, tokens=t, dtype=dtype, flags=flags, scale=scale)
    out, lse, status = run(c, p, q)
    assert status == b.GRKV_OK
    check(c, q64, out, lse, [t] * 4, scale)


# Logits past fp32's range are infinite and make their row NaN.  Not so in the tensor-core kernel of bf16 with 17 rows
# and more, whose products with the scale are not rounded and whose references are rounded down (at most fp32's largest
# number): there such slots weigh the same.
@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
def test_logits_past_the_range(grkv_lib, dtype, flags, g, t):
    """No row passes for one that sees nothing."""
    c = R.Cache([300, 65], 32, dtype, 72)
    q, q64 = queries(2, g, t, dtype, 73)
    p = b.cache_params(2, g, c.pages, 32, c.cols, tokens=t, dtype=dtype, flags=flags, scale=2.0 ** 127)
    for u in range(2):                           # every row has a logit past 2^128
        assert ((q64[u] @ c.slots(u)[0].T).max(-1) > 4).all()
    out, lse, _ = run(c, p, q)
    if dtype == "bf16" and not flags and g * t > 16:
        assert torch.isfinite(out).all() and torch.isfinite(lse).all() and (lse > 2.0 ** 126).all()
    else:
        assert torch.isnan(out).all() and not torch.isfinite(lse).any() and not (lse == -math.inf).any()
