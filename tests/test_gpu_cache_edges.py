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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_units_than_a_grid_has_rows(grkv_lib, dtype):
    """Every page operator over 70000 units (grids of 65535 rows go round), then attention."""
    units, page, cols, spare = 70000, 16, 2, 9
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 2 * page, units).astype(np.int32)
    want = np.minimum(lens + rng.integers(0, 3, units), cols * page).astype(np.int32)
    pages = units * cols + spare
    dt = R.TORCH[dtype]
    p = b.cache_params(units, 2, pages, page, cols, tokens=2, dtype=dtype)
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    ok = lambda: b.grkv_status(ws) == b.GRKV_OK
    dk, dv = (torch.zeros(pages, page, D, dtype=dt, device="cuda") for _ in range(2))
    table = torch.full((units, cols), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    zero, dl, dw = torch.zeros(units, dtype=torch.int32, device="cuda"), R.int_dev(lens), R.int_dev(want)
    for have, to in ((zero, dl), (dl, dw)):
        b.grkv_cache_reserve(p, table, have, to, refs, dk, dv, ws)
        assert ok()
    t_ref, r_ref = np.full((units, cols), -1, np.int32), np.zeros(pages, np.int32)
    none = np.zeros((pages, 1, 1))
    assert R.reserve(t_ref, np.zeros(units, int), lens, r_ref, none, none, page)
    assert R.reserve(t_ref, lens, want, r_ref, none, none, page)
    assert np.array_equal(table.cpu().numpy(), t_ref) and np.array_equal(refs.cpu().numpy(), r_ref)
    # a row's elements say whose it is; its values, which of the unit's
    slot = torch.arange(cols * page, device="cuda")
    at = (table.long().clamp_min(0)[:, slot // page] * page + slot % page)
    live = slot[None] < dw[:, None]
    dk.view(-1, D)[at[live]] = (torch.arange(units, device="cuda") % 61)[:, None].expand_as(live)[live][:, None].to(dt)
    dv.view(-1, D)[at[live]] = slot[None].expand_as(live)[live][:, None].to(dt)
    new = torch.full((units, 2, D), 40, dtype=dt, device="cuda")
    count = dw - dl
    b.grkv_cache_append(p, new, new, dk, dv, table, dw, ws, count=count)
    assert ok()
    got = dv.view(-1, D)[at][..., 5].float()
    assert torch.equal(got[live], torch.where(slot[None] >= dl[:, None], 40.0, slot[None].float())[live])
    # equal logits: the mean of a unit's values
    q = torch.zeros(units, 2, 1, D, dtype=dt, device="cuda")
    p1 = b.cache_params(units, 2, pages, page, cols, dtype=dtype)
    out = torch.full_like(q, 7)
    b.grkv_attend(p1, q, dk, dv, table, dw, out, ws)
    assert ok()
    total = (torch.where(live, got, 0.0)).double().sum(1)
    mean = torch.where(dw > 0, total / dw.clamp_min(1), 0.0)
    assert ((out[:, :, 0, 77].double() - mean[:, None]).abs() <= mean[:, None] * (2.0 ** -8 + 2.0 ** -19)).all()
    # the last slot of every unit to its first place, then the fork of all and the end of all
    keep = (dw > 0).int()
    b.grkv_cache_compact(p1, (dw - 1).clamp_min(0)[:, None].contiguous(), dk, dv, table, dw, table, ws, keep=keep)
    assert ok()
    has = dw > 0
    last = got.gather(1, (dw.long() - 1).clamp_min(0)[:, None])[:, 0]
    assert torch.equal(dv.view(-1, D)[at[:, 0]][:, 127].float()[has], last[has])
    t2, l2 = torch.empty_like(table), torch.empty_like(dw)
    b.grkv_cache_fork(p1, torch.arange(units, device="cuda").flip(0).int(), table, keep, t2, l2, refs, ws)
    assert ok()
    assert torch.equal(l2, keep.flip(0)) and torch.equal(t2[:, 0], torch.where(keep > 0, table[:, 0], -1).flip(0))
    for tb in (table, t2):
        b.grkv_cache_trim(p1, tb, zero, refs, ws)
        assert ok() and (tb == -1).all()
    assert (refs == 0).all()


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("f32", 0)])
def test_a_captured_step_is_replayed(grkv_lib, dtype, flags):
    """Reserve, append, attention and the lengths' step in one graph, replayed token after token, against
    the same calls made one by one; other work of the same kind runs beside it."""
    units, g, page, cols, steps = 6, 4, 16, 6, 20
    start = [0, 15, 16, 31, 40, 63]
    dt = R.TORCH[dtype]
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float32, device="cuda", generator=gen).to(dt)
    kn, vn, qn = rnd(steps, units, 1, D), rnd(steps, units, 1, D), rnd(steps, units, g, 1, D)
    pages = units * cols
    p = b.cache_params(units, g, pages, page, cols, dtype=dtype, flags=flags)
    k0, v0 = rnd(pages, page, D), rnd(pages, page, D)

    class Side:
        def __init__(self):
            self.k, self.v = k0.clone(), v0.clone()
            self.table = torch.full((units, cols), -1, dtype=torch.int32, device="cuda")
            self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
            self.lens, self.now = R.int_dev(start), torch.zeros(units, dtype=torch.int32, device="cuda")
            self.ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
            self.x = [torch.empty_like(t[0]) for t in (kn, vn, qn)]
            self.out = torch.zeros_like(qn[0])
            b.grkv_cache_reserve(p, self.table, torch.zeros_like(self.lens), self.lens, self.refs, self.k,
                                 self.v, self.ws)
            assert b.grkv_status(self.ws) == b.GRKV_OK

        def step(self):
            torch.add(self.lens, 1, out=self.now)
            b.grkv_cache_reserve(p, self.table, self.lens, self.now, self.refs, self.k, self.v, self.ws)
            b.grkv_cache_append(p, self.x[0], self.x[1], self.k, self.v, self.table, self.now, self.ws)
            b.grkv_attend(p, self.x[2], self.k, self.v, self.table, self.now, self.out, self.ws)
            self.lens.copy_(self.now)

        def feed(self, i):
            for to, t in zip(self.x, (kn, vn, qn)):
                to.copy_(t[i])

    eager, graphed, beside = Side(), Side(), Side()
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        graphed.step()
    torch.cuda.synchronize()
    for i in range(steps):
        for side in (eager, graphed, beside):
            side.feed(i)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            beside.step()
        with torch.cuda.stream(stream):
            graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for side in (graphed, beside):
            assert torch.equal(side.out, eager.out) and torch.equal(side.table, eager.table)
            assert torch.equal(side.lens, eager.lens) and torch.equal(side.refs, eager.refs)
    for side in (eager, graphed, beside):
        assert b.grkv_status(side.ws) == b.GRKV_OK
    assert torch.equal(graphed.k, eager.k) and torch.equal(graphed.v, eager.v)
    u = 3
    rows = eager.table[u].long().repeat_interleave(page) * page + torch.arange(cols * page, device="cuda") % page
    n = start[u] + steps
    kk, vv = (t.view(-1, D)[rows[:n]].double().cpu().numpy() for t in (eager.k, eager.v))
    o, _, mass, err = R.attend_unit(qn[-1, u].double().cpu().numpy(), kk, vv, 1, 0, 4)
    tol = (2 * err + 2.0 ** -13 + 2.0 ** -8)[..., None] * mass + 2.0 ** -8 * np.abs(o)
    assert (np.abs(eager.out[u].double().cpu().numpy() - o) <= tol).all()
