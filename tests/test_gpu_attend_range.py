"""grkv_attend where logits, or values times probabilities, are near the ends of what fp32 holds."""
import math

import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
D = R.D
TYPES = [("f32", 0), ("bf16", 0), ("bf16", b.GRKV_FORCE_SIMT)]
# heads, tokens: items of 5, 12, 50, 100 and 300 rows (every kernel and form of the tensor cores' tile)
ROWS = [(5, 1), (6, 2), (50, 1), (50, 2), (60, 5)]


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("power", [22, 26, 31, 40, 100])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("late", [False, True])
def test_finite_logits_of_any_size(grkv_lib, dtype, flags, g, t, power, sign, late):
    """Logits of about +-2^power beside ordinary ones in the same tile.  Queries and keys have one
    element that is not zero, of 8 bits, so that fp32 holds every product exactly; the largest
    logit of a unit is apart from the next by 2^-5 of itself, so its slot (or the two that
    share it) has all the weight.  Units of 6 slot tiles, many more than there are CTAs, with that
    slot in the first tile, in the last, or in both.  late: the first 300 slots' logits are ordinary ones
    (below all others if those are positive, the largest if they are negative)."""
    n, page, units = 700, 64, 420
    rng = np.random.default_rng(power)
    cols = R.pages_of(n, page)
    key = 1 + rng.integers(4, 120, (3, n)) / 128.0           # in [1 + 2^-5, 2 - 2^-4]
    top = 1 if sign < 0 else 2 - 1 / 128                     # the largest times a query below or above 0
    for c, slots in enumerate(([317 if late else 17], [680], [340 if late else 40, 690])):
        key[c, slots] = top
    if late:
        key[:, :300] *= 2.0 ** -power
    head = 1 + rng.integers(0, 128, (units, g, t)) / 128.0
    head *= sign * 2.0 ** (power // 2)
    plain = rng.random((units, g, t)) < 0.25                 # ordinary logits
    head[plain] = rng.integers(-64, 65, plain.sum()) / 16.0 * 2.0 ** -(power - power // 2)
    key *= 2.0 ** (power - power // 2)
    dt = R.TORCH[dtype]
    gen = torch.Generator(device="cuda").manual_seed(power)
    k = torch.zeros(3 * cols * page, D, dtype=torch.float64, device="cuda")
    k.view(3, cols * page, D)[:, :n, 77] = torch.from_numpy(key).cuda()
    v = torch.randn(3 * cols * page, D, dtype=torch.float32, device="cuda", generator=gen).to(dt)
    q = torch.zeros(units, g, t, D, dtype=torch.float64, device="cuda")
    q[..., 77] = torch.from_numpy(head).cuda()
    table = (torch.arange(units, device="cuda")[:, None] % 3 * cols
             + torch.arange(cols, device="cuda")[None]).int().contiguous()
    lens = torch.full((units,), n, dtype=torch.int32, device="cuda")
    p = b.cache_params(units, g, 3 * cols, page, cols, tokens=t, dtype=dtype, flags=flags)
    out = torch.zeros(units, g, t, D, dtype=dt, device="cuda")
    lse = torch.zeros(units, g, t, dtype=torch.float32, device="cuda")
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    b.grkv_attend(p, q.to(dt), k.to(dt), v, table, lens, out, ws, lse=lse)
    assert b.grkv_status(ws) == b.GRKV_OK
    s = 1 / math.sqrt(D)
    see = torch.arange(n, device="cuda")[None] <= n - t + torch.arange(t, device="cuda")[:, None]
    for c in range(3):
        x = q[c::3, ..., 77:78] * k.view(3, -1, D)[c, :n, 77] * s
        x = x.masked_fill(~see, -math.inf)
        vv = v.view(3, -1, D)[c, :n].double()
        w = torch.softmax(x, -1)
        o, mass, z = w @ vv, w @ vv.abs(), torch.logsumexp(x, -1)
        # Ordinary logits: |x| < 0.09 x 4 x 2, off by 4 u of itself; the others' weights are 0 or
        # shared, whatever the logits' last bits.  Then the exponential, n fp32 sums, P in bf16.
        rel = 2 * 4 * R.U32 * 0.75 + (n + 64) * R.U32 + 2.0 ** -21
        tol = (rel + (2.0 ** -8 if dtype == "bf16" else 0)) * mass + R.ROUND[dtype] * o.abs()
        off = (out[c::3].double() - o).abs()
        assert (off <= tol).all(), f"cache {c}: {(~(off <= tol)).sum().item()} off"
        # scale, product, ln 2 and the sum: 8 roundings of lse itself
        assert ((lse[c::3].double() - z).abs() <= 8 * R.U32 * z.abs() + rel).all()


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
def test_many_tiles_of_large_probabilities(grkv_lib, dtype, flags, g, t):
    """Outputs before their division stay within 2^60 times the values for a whole run of tiles.  Units of
    1200 slot tiles, a few to a CTA: the first tile's logits are 0, all others' 52.5 log2 units above,
    2^59.5 a tile, and their values 2^59: 1200 such tiles would be 2^128.7."""
    tiles, page, units = 1200, 128, 304
    n, dt = tiles * page, R.TORCH[dtype]
    k = torch.zeros(2, page, D, dtype=dt, device="cuda")
    v = torch.ones(2, page, D, dtype=dt, device="cuda")
    k[1, :, 3], v[1] = 7, 2.0 ** 59
    q = torch.zeros(units, g, t, D, dtype=dt, device="cuda")
    q[..., 3] = 7.5
    table = torch.ones(units, tiles, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    lens = torch.full((units,), n, dtype=torch.int32, device="cuda")
    p = b.cache_params(units, g, 2, page, tiles, tokens=t, dtype=dtype, flags=flags,
                       scale=math.log(2.0))
    out, lse = torch.zeros_like(q), torch.zeros(units, g, t, dtype=torch.float32, device="cuda")
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    b.grkv_attend(p, q, k, v, table, lens, out, ws, lse=lse)
    assert b.grkv_status(ws) == b.GRKV_OK
    # logits are exact, the scale 2 u off: 2 x 37 x 2 u a probability; n fp32 sums; P and out in bf16
    rel = 2 * 37 * 2 * R.U32 + (n + 64) * R.U32 + 2.0 ** -21
    tol = rel + (2.0 ** -8 if dtype == "bf16" else 0) + R.ROUND[dtype]
    assert ((out.double() / 2.0 ** 59 - 1).abs() <= tol).all()
    seen = n - t + 1 + torch.arange(t, device="cuda", dtype=torch.float64) - page
    z = torch.log(seen * 2.0 ** 52.5 + page)
    assert ((lse.double() - z).abs() <= rel + 4 * R.U32 * z).all()
