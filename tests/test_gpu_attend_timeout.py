"""The exit of the attention's bounded waits (grkv_attend on the tensor cores)."""
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
D = R.D


# items of 5 rows (one tile, both parts of P), of 100 (one tile) and of 256 (two tiles); masked tiles
# at the ends of runs, or at windows in every item
@pytest.mark.parametrize("g,t,window", [(5, 1, 0), (50, 2, 0), (50, 2, 300), (4, 200, 0), (4, 200, 300)])
def test_a_wait_that_runs_out_ends_the_call(grkv_lib, g, t, window):
    """GRKV_TEST_TIMEOUT: a warp of the first CTA's search of V withholds one arrive, and waits for its
    next tiles for about 2 ms only.  Every role of that CTA gives up; loads and products under
    way end, tensor memory is freed, the call returns and the status says GRKV_ERR_TIMEOUT.
    The calls after it, in the same workspace, give what the one before gave."""
    units, page, cols = 300, 64, 60
    gen = torch.Generator(device="cuda").manual_seed(g)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float32, device="cuda", generator=gen).bfloat16()
    k, v, q = rnd(cols, page, D), rnd(cols, page, D), rnd(units, g, t, D)
    table = torch.arange(cols, device="cuda").int().repeat(units, 1)
    lens = torch.full((units,), cols * page - 5, dtype=torch.int32, device="cuda")
    p = b.cache_params(units, g, cols, page, cols, tokens=t, window=window)
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    outs = []
    for flags in (0, b.GRKV_TEST_TIMEOUT, 0, b.GRKV_TEST_TIMEOUT, 0):
        p.flags = flags
        out = torch.zeros_like(q)
        b.grkv_attend(p, q, k, v, table, lens, out, ws)
        assert b.grkv_status(ws) == (b.GRKV_ERR_TIMEOUT if flags else b.GRKV_OK)
        if not flags:
            outs.append(out)
    assert outs[0].abs().max() > 0
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_the_cuda_core_kernels_have_no_such_waits(grkv_lib):
    p = b.cache_params(1, 2, 4, 64, 4, flags=b.GRKV_TEST_TIMEOUT | b.GRKV_FORCE_SIMT)
    pool = torch.ones(4, 64, D, dtype=torch.bfloat16, device="cuda")
    q = torch.ones(1, 2, 1, D, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    b.grkv_attend(p, q, pool, pool, R.int_dev([[0, 1, 2, 3]]), R.int_dev([200]), out, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
    assert (out == 1).all()
