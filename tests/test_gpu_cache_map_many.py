"""Positions and slots of as many packed units as a call takes, whose first rows a kernel of its own sums up."""
import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as C

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("u,t", [(1 << 20, 3), ((1 << 20) - 1, 1), (300000, 40)])
def test_many_packed_units(grkv_lib, u, t):
    rng = np.random.default_rng(t)
    page, cols = 16, 4
    lens = rng.integers(t, cols * page + 1, u)
    count = rng.integers(0, t + 1, u)
    offset = rng.integers(0, 1000, u)
    pages = 1 << 22
    table = rng.integers(0, pages, (u, cols))     # any pages: nothing is written to them
    p = b.cache_params(u, 1, pages, page, cols, tokens=t)
    ws = torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")
    pos = torch.full((u, t), 77, dtype=torch.int32, device="cuda")
    slot = torch.full((u, t), 77, dtype=torch.int64, device="cuda")
    first = torch.full((u + 1,), 77, dtype=torch.int64, device="cuda")
    b.grkv_cache_map(p, C.int_dev(table), C.int_dev(lens), pos, slot, ws, count=C.int_dev(count),
                     offset=C.int_dev(offset), first_row=first)
    assert b.grkv_status(ws) == b.GRKV_OK
    want = np.concatenate([[0], np.cumsum(count)])
    assert np.array_equal(first.cpu().numpy(), want)
    unit = np.repeat(np.arange(u), count)
    s = lens[unit] - count[unit] + np.arange(want[-1]) - want[unit]
    tail = np.full(u * t - want[-1], -1)
    assert np.array_equal(pos.cpu().numpy().ravel(), np.concatenate([s + offset[unit], tail]))
    row = table[unit, s // page] * page + s % page
    assert np.array_equal(slot.cpu().numpy().ravel(), np.concatenate([row, tail]))
