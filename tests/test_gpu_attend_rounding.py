"""Large logits in every instance of the kernels that take exponents from rounded logits: a product that is not
rounded as its reference was would weigh a row's largest slot 2^256 and more."""
import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R
from tests.test_gpu_attend import TYPES, queries, workspace

pytestmark = pytest.mark.gpu
ROWS = [(1, 1), (2, 1), (1, 2), (3, 1), (4, 1), (1, 4), (5, 1), (8, 1), (9, 1), (3, 4), (16, 1), (4, 4), (20, 1), (4, 90)]


# Logits of 2^29 to 2^125 leave every row its largest one's value, where that is clear: by 2^-10 of the largest, a
# thousand times what fp32 sums of 128 products lose (130 x 2^-24).
@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("cross", [True, False])
def test_the_largest_slot_takes_all(grkv_lib, dtype, flags, g, t, cross):
    c = R.Cache([700, 90], 64, dtype, 80)
    q, q64 = queries(2, g, t, dtype, 81)
    p = b.cache_params(2, g, c.pages, 64, c.cols, tokens=t, dtype=dtype, flags=flags)
    kd, vd = c.dev()
    dq, table, lens, ws = q.cuda(), R.int_dev(c.table), R.int_dev(c.lens), workspace(p)
    for power in (24, 30, 40, 70, 120):
        p.scale = 2.0 ** power
        out, lse = torch.zeros_like(dq), torch.zeros(q.shape[:3], dtype=torch.float32, device="cuda")
        (b.grkv_attend_cross if cross else b.grkv_attend)(p, dq, kd, vd, table, lens, out, ws, lse=lse)
        assert b.grkv_status(ws) == b.GRKV_OK and torch.isfinite(out).all() and torch.isfinite(lse).all()
        for u, n in enumerate(c.lens):
            k, v = c.slots(u)
            x = q64[u] @ k.T
            if not cross:                        # the last t slots are the rows' own
                x = np.where(np.arange(n) <= n - t + np.arange(t)[:, None], x, -np.inf)
            top = np.sort(x, -1)
            clear = top[..., -1] - top[..., -2] > 2.0 ** -10 * top[..., -1]
            want = v[x.argmax(-1)]
            off = np.abs(out[u].double().cpu().numpy() - want)
            assert clear.mean() > 0.5 and (off <= R.ROUND[dtype] * np.abs(want))[clear].all()
