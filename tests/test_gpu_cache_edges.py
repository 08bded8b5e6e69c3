"""The paged cache's page operators where tables have holes, end, or are long."""
import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R
from tests.test_gpu_cache import Dev

pytestmark = pytest.mark.gpu
D = R.D


@pytest.mark.parametrize("cols", [12, 200])
def test_units_without_their_first_pages_are_forked(grkv_lib, cols):
    """Pages in front of every window may be gone, for attention and for a fork: a column without
    a page has none in the fork either.  (One block that writes the status itself, and many.)"""
    page, units = 16, 30
    rng = np.random.default_rng(1)
    c = R.Cache([int(x) for x in rng.integers(100, 11 * page, units)], page, "bf16", 2, spare=9)
    c.table = np.concatenate([c.table, np.full((units, cols - c.cols), -1, np.int32)], 1)
    c.cols = cols
    for u in range(0, units, 2):
        for col in range(1, 1 + u % 5):     # the sinks' page stays, those behind it are gone
            c.refs[c.table[u, col]] -= 1
            c.table[u, col] = -1 if u % 4 else -2 ** 31
    src = [int(x) for x in rng.integers(-1, units, 17)]
    d = Dev(c)
    p = b.cache_params(len(src), 2, c.pages, page, cols)
    table = torch.full((len(src), cols), 7, dtype=torch.int32, device="cuda")
    lens = torch.full((len(src),), 7, dtype=torch.int32, device="cuda")
    b.grkv_cache_fork(p, R.int_dev(src), d.table, d.lens, table, lens, d.refs, d.ws)
    d.ok()
    want = np.full((len(src), cols), -1, np.int32)
    for u, s in enumerate(src):
        m = R.pages_of(c.lens[s], page) if s >= 0 else 0
        want[u, :m] = np.maximum(c.table[s, :m], -1)
        np.add.at(c.refs, want[u][want[u] >= 0], 1)
    assert np.array_equal(table.cpu().numpy(), want)
    assert lens.tolist() == [c.lens[s] if s >= 0 else 0 for s in src]
    d.same()
    # an entry behind the pool is still reported, and taken as none
    d.table[src[0] if src[0] >= 0 else 0, 0] = c.pages
    c.table[src[0] if src[0] >= 0 else 0, 0] = c.pages
    before = d.refs.clone()
    b.grkv_cache_fork(p, R.int_dev([max(src[0], 0)] + [-1] * (len(src) - 1)), d.table, d.lens, table,
                      lens, d.refs, d.ws)
    d.ok(b.GRKV_ERR_INVALID_ARG)
    assert table[0, 0].item() == -1 and (table[0] >= 0).sum().item() == (d.refs - before).sum().item()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_behind_a_full_table_are_not_written_over_others(grkv_lib, dtype):
    """A length past the table: rows that have a slot go there, the others nowhere."""
    page, t = 16, 5
    c = R.Cache([96, 95, 96, 40, 96], page, dtype, 3)
    cap = c.cols * page
    assert cap == 96
    rng = np.random.default_rng(4)
    kn, vn = (c.rounded(rng.standard_normal((5, t, D))) for _ in range(2))
    d = Dev(c, tokens=t)
    as_t = lambda x: torch.from_numpy(x).to(R.TORCH[dtype]).cuda()
    lens, count = [97, 98, 2 ** 31 - 1, 40, 101], [1, 3, 5, 2, 5]
    b.grkv_cache_append(d.p, as_t(kn), as_t(vn), d.k, d.v, d.table, R.int_dev(lens), d.ws,
                        count=R.int_dev(count))
    d.ok(b.GRKV_ERR_INVALID_ARG)
    for u, (n, m) in enumerate(zip(lens, count)):
        for i in range(m):
            if n - m + i < cap:
                at = R.at(c.table, u, n - m + i, page)
                c.k[at], c.v[at] = kn[u, i], vn[u, i]
    d.same()


@pytest.mark.parametrize("units,page", [(1, 16), (7, 16), (60, 32), (1024, 16), (1500, 16)])
def test_reserve_of_many_columns(grkv_lib, units, page):
    """A prompt's or a compressed cache's first reserve, and more than 32 columns behind shared pages:
    decisions are marked in the table whatever the number of units."""
    rng = np.random.default_rng(units)
    cols = 90 if units <= 60 else 40
    lens = rng.integers(0, 30 * page, units)
    lens[::3] = 0
    want = np.minimum(lens + rng.integers(0, (cols - 30) * page, units), cols * page)
    want[0] = cols * page
    table = np.full((units, cols), -1, np.int32)
    pages = units * cols + 50
    order = rng.permutation(pages)
    at = 0
    for u in range(units):
        m = R.pages_of(int(lens[u]), page)
        table[u, :m] = order[at:at + m]
        at += m
        if u % 4 == 1 and m:        # a fork of the unit before: shares what that one has
            p = R.pages_of(int(lens[u - 1]), page)
            lens[u] = min(lens[u - 1], want[u])
            table[u] = -1
            table[u, :R.pages_of(int(lens[u]), page)] = table[u - 1, :R.pages_of(int(lens[u]), page)]
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    refs[rng.integers(0, pages, 20)] += 1                    # another table's
    k = rng.integers(-50, 50, (pages, page, 4)).astype(np.float64)
    v = k + 1
    p = b.cache_params(units, 1, pages, page, cols)
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    dk, dv = (torch.from_numpy(np.repeat(x, 32, 2)).bfloat16().cuda() for x in (k, v))
    dt, dr = R.int_dev(table), R.int_dev(refs)
    b.grkv_cache_reserve(p, dt, R.int_dev(lens), R.int_dev(want), dr, dk, dv, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
    assert R.reserve(table, lens, want, refs, k, v, page)
    assert np.array_equal(dt.cpu().numpy(), table) and np.array_equal(dr.cpu().numpy(), refs)
    assert np.array_equal(dk.double().cpu().numpy(), np.repeat(k, 32, 2))
    assert np.array_equal(dv.double().cpu().numpy(), np.repeat(v, 32, 2))
