"""Rotary positions of rows, appended and kept keys against 64-bit formulas."""
import math

import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as C
from tests import rope_ref as R

pytestmark = pytest.mark.gpu
D = C.D
TYPES = ["bf16", "f32"]
ROTARY = [2, 10, 48, 50, 64, 126, 128]


def plan(layout="half", **kw):
    return b.grkv_rope_make(b.rope_params(layout=layout, **kw))


def normal(rng, dtype, *shape):
    return torch.from_numpy(rng.standard_normal(shape)).to(C.TORCH[dtype])


def host(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rotary", ROTARY)
@pytest.mark.parametrize("transpose", [False, True])
def test_rows(grkv_lib, dtype, layout, rotary, transpose):
    """Positions from 0 to the largest, padding left as it was."""
    rng = np.random.default_rng(rotary)
    kw = dict(rotary=rotary, scaling="yarn", factor=3.0, original=2048.0)
    x = normal(rng, dtype, 3, 5, 7, D)
    pos = rng.integers(0, 1 << 31, (3, 7))
    pos[0, :4] = [0, 1, 2, 2 ** 31 - 1]
    pos[1, 2] = pos[2, 6] = -1
    out = torch.full((3, 5, 7, D), 7.0, dtype=C.TORCH[dtype], device="cuda")
    b.grkv_rope_rows(plan(layout, **kw), x.cuda(), out, pos=C.int_dev(pos), transpose=transpose)
    want, err = R.rotate(x.double().numpy(), pos[:, None], layout, transpose, dtype=dtype, **kw)
    skip = np.broadcast_to((pos < 0)[:, None, :, None], want.shape)
    want, err = np.where(skip, 7.0, want), np.where(skip, 0.0, err)
    R.check(host(out), want, err, dtype)
    assert torch.equal(out[..., rotary:].cpu()[~torch.from_numpy(skip[..., rotary:].copy())],
                       x[..., rotary:][~torch.from_numpy(skip[..., rotary:].copy())])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("s,h,t", [(1, 1, 1), (1, 33, 1), (70, 1, 1), (2, 9, 65), (1, 2, 1031), (5, 40, 3)])
def test_sizes_and_starts(grkv_lib, dtype, s, h, t):
    rng = np.random.default_rng(s * h + t)
    x = normal(rng, dtype, s, h, t, D)
    start = rng.integers(0, 1 << 20, s)
    start[0] = 0
    p = start[:, None] + np.arange(t)
    for name in ("start", "pos", None):
        kw = {"start": C.int_dev(start), "pos": C.int_dev(p)}.get(name)
        out = torch.empty(s, h, t, D, dtype=C.TORCH[dtype], device="cuda")
        b.grkv_rope_rows(plan("pairs"), x.cuda(), out, **({name: kw} if name else {}))
        at = p if name else np.broadcast_to(np.arange(t), (s, t))
        R.check(host(out), *R.rotate(x.double().numpy(), at[:, None], "pairs", dtype=dtype), dtype)


def test_starts_before_the_first_token_and_past_the_last_position(grkv_lib):
    x = normal(np.random.default_rng(1), "f32", 2, 1, 9, D)
    out = torch.full((2, 1, 9, D), 7.0, dtype=torch.float32, device="cuda")
    b.grkv_rope_rows(plan(), x.cuda(), out, start=C.int_dev([-4, 2 ** 31 - 3]))
    p = np.array([[-4], [2 ** 31 - 3]]) + np.arange(9)      # not wrapped around
    want, err = R.rotate(x.double().numpy(), p[:, None])
    want[0, :, :4], err[0, :, :4] = 7.0, 0.0
    R.check(host(out), want, err, "f32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout,rotary", [("half", 128), ("half", 36), ("pairs", 20)])
def test_strides(grkv_lib, dtype, layout, rotary):
    """The query part of a projection's output [S][t][3 H][D], one head for all, in place."""
    rng = np.random.default_rng(3)
    s, h, t = 2, 6, 19
    rope = plan(layout, rotary=rotary)
    whole = normal(rng, dtype, s, t, 3 * h, D).cuda()
    x = whole[:, :, h:2 * h].transpose(1, 2)
    pos = rng.integers(0, 5000, (s, t))
    want, err = R.rotate(host(x), pos[:, None], layout, rotary=rotary, dtype=dtype)
    out = torch.empty(s, h, t, D, dtype=x.dtype, device="cuda")
    b.grkv_rope_rows(rope, x, out, pos=C.int_dev(pos))
    R.check(host(out), want, err, dtype)
    back = torch.zeros(s, t, h, D, dtype=x.dtype, device="cuda")       # and into the projection's
    b.grkv_rope_rows(rope, x, back.transpose(1, 2), pos=C.int_dev(pos))
    assert torch.equal(back.transpose(1, 2), out)
    one = x[:, 2:3].expand(s, h, t, D)
    b.grkv_rope_rows(rope, one, back.transpose(1, 2), pos=C.int_dev(pos))
    assert torch.equal(back.transpose(1, 2), out[:, 2:3].expand(s, h, t, D))
    before = whole.clone()
    b.grkv_rope_rows(rope, x, x, pos=C.int_dev(pos))
    assert torch.equal(x, out)
    before[:, :, h:2 * h] = x.transpose(1, 2)
    assert torch.equal(whole, before)                                    # the other heads stay


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rotary", [20, 64])
def test_values_that_are_not_finite_stay_in_their_pair(grkv_lib, dtype, layout, rotary):
    rng = np.random.default_rng(5)
    x = normal(rng, dtype, 1, 1, 4, D)
    i, j = R.pairs(rotary, layout)
    x[0, 0, 0, int(i[3])], x[0, 0, 1, int(j[rotary // 2 - 1])] = math.nan, math.inf
    x[0, 0, 2, rotary:] = math.nan
    x[0, 0, 3, rotary], x[0, 0, 3, 127] = math.inf, -math.inf
    out = torch.empty(1, 1, 4, D, dtype=x.dtype, device="cuda")
    b.grkv_rope_rows(plan(layout, rotary=rotary), x.cuda(), out, start=C.int_dev([17]))
    got, want = host(out), R.rotate(x.double().numpy(), 17 + np.arange(4)[None, None], layout, rotary=rotary)[0]
    hit = np.zeros(got.shape, bool)
    for row, k in ((0, 3), (1, rotary // 2 - 1)):
        hit[0, 0, row, [i[k], j[k]]] = True
    assert not np.isfinite(got[hit]).any()
    assert np.array_equal(got[..., rotary:], x.double().numpy()[..., rotary:], equal_nan=True)
    fine = ~hit
    fine[..., rotary:] = False
    assert np.allclose(got[fine], want[fine], atol=0.05)


@pytest.mark.parametrize("layout,rotary", [("half", 128), ("half", 18), ("pairs", 30)])
def test_the_transposed_product_is_the_gradient(grkv_lib, layout, rotary):
    """Against the forward's differences: it is linear, so over steps of any size, here of ones."""
    rope = plan(layout, rotary=rotary, amplitude=1.25)
    rng = np.random.default_rng(7)
    up = normal(rng, "f32", 1, 1, 1, D).cuda()
    grad, zero = torch.empty_like(up), torch.zeros(1, 1, 1, D, dtype=torch.float32, device="cuda")
    b.grkv_rope_rows(rope, up, grad, start=C.int_dev([777]), transpose=True)
    eye = torch.eye(D, dtype=torch.float32, device="cuda").view(1, D, 1, D).contiguous()
    moved, base = torch.empty_like(eye), torch.empty_like(zero)
    b.grkv_rope_rows(rope, eye, moved, start=C.int_dev([777]))
    b.grkv_rope_rows(rope, zero, base, start=C.int_dev([777]))
    diff = ((moved - base).double() * up.double()).sum(-1).view(D)
    # both sides: two products of values off by BIG, of |up| < 5
    assert (grad.double().view(D) - diff).abs().max() < 2 * 2 * 5 * 1.25 * (R.BIG + 2.0 ** -24)


def test_rows_further_apart_than_32_bits(grkv_lib):
    n = (1 << 31) + 1024
    x = torch.zeros(n + D, dtype=torch.bfloat16, device="cuda")
    rows = x.as_strided((1, 2, 1, D), (0, n, 0, 1))
    rows.normal_()
    want, err = R.rotate(host(rows), np.full((1, 2, 1), 99), "half", dtype="bf16")
    b.grkv_rope_rows(plan(), rows, rows, start=C.int_dev([99]))
    R.check(host(rows), want, err, "bf16")


def test_graphs_and_streams(grkv_lib):
    rng = np.random.default_rng(8)
    x = normal(rng, "bf16", 4, 8, 33, D).cuda()
    rope, out, direct = plan(), torch.zeros_like(x), torch.zeros_like(x)
    start = C.int_dev([5, 6, 7, 8])
    b.grkv_rope_rows(rope, x, direct, start=start)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.grkv_rope_rows(rope, x, out, start=start)
    rope.amplitude = 3.0                       # the plan was read when the call was made
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, direct)
    start.add_(1)                              # positions are read when it runs
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(out, direct)
    rope.amplitude = 1.0
    with torch.cuda.stream(side):
        b.grkv_rope_rows(rope, x, direct, start=start)
    side.synchronize()
    assert torch.equal(out, direct)


# ------------------------------------------------------------------------ append
class Dev:
    """A cache on the device beside its copy in numpy."""

    def __init__(self, c, g, tokens):
        self.c, self.p = c, b.cache_params(len(c.lens), g, c.pages, c.page, c.cols, tokens=tokens,
                                           dtype=c.dtype)
        self.k, self.v = c.dev()
        self.table, self.lens = C.int_dev(c.table), C.int_dev(c.lens)
        self.ws = torch.full((b.grkv_cache_workspace_size(self.p),), 0xFF, dtype=torch.uint8, device="cuda")

    def same(self, err_k, code=b.GRKV_OK):
        assert b.grkv_status(self.ws) == code
        got, c = host(self.k), self.c
        assert np.array_equal(np.isnan(got), np.isnan(c.k))
        fine = ~np.isnan(got)
        R.check(got[fine], c.k[fine], err_k[fine], c.dtype)
        assert np.array_equal(host(self.v), c.v, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout,rotary", [("half", 128), ("half", 64), ("half", 12), ("pairs", 128),
                                           ("pairs", 22)])
@pytest.mark.parametrize("g,t,page", [(1, 1, 16), (4, 1, 64), (5, 40, 32), (8, 9, 128), (64, 2, 16)])
@pytest.mark.parametrize("where", ["slots", "offset", "pos", "packed"])
def test_append(grkv_lib, dtype, layout, rotary, g, t, page, where):
    """New rows of units of uneven lengths, with counts and without, by unit and packed."""
    rng = np.random.default_rng(g * t)
    c = C.Cache([t, t + 15, 200, t + 100, 333], page, dtype, g + t, extra_cols=1)
    u = len(c.lens)
    d = Dev(c, g, t)
    kw = dict(rotary=rotary, scaling="bands", factor=4.0, amplitude=1.5)
    count = [t] * u if where == "slots" else [int(x) for x in rng.integers(0, t + 1, u)]
    if where == "pos":
        count[2] = 0
    offset = rng.integers(0, 1 << 30, u) if where == "offset" else np.zeros(u, int)
    n = sum(count) + 7 if where == "packed" else u * t
    first = np.array([sum(count[:x]) + 3 if where == "packed" else x * t for x in range(u)])
    k_new, v_new = normal(rng, dtype, n, D), normal(rng, dtype, n, D)
    given = rng.integers(0, 1 << 21, n)
    q = normal(rng, dtype, u, g, t, D)
    q_out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    args = dict(q=q.cuda(), q_out=q_out)
    if where != "slots":
        args["count"] = C.int_dev(count)
    if where == "offset":
        args["offset"] = C.int_dev(offset)
    if where in ("pos", "packed"):
        args["pos"] = C.int_dev(given)
    if where == "packed":
        args["first_row"] = torch.from_numpy(first).cuda()
    b.grkv_cache_append_rope(d.p, plan(layout, **kw), k_new.cuda(), v_new.cuda(), d.k, d.v, d.table,
                             d.lens, d.ws, **args)
    err = np.zeros_like(c.k)
    want_q, err_q = np.full(q.shape, 7.0), np.zeros(q.shape)
    for x in range(u):
        for i in range(count[x]):
            slot = c.lens[x] - count[x] + i
            at, row = C.at(c.table, x, slot, page), first[x] + i
            p = given[row] if where in ("pos", "packed") else slot + offset[x]
            c.k[at], err[at] = R.rotate(k_new[row].double().numpy(), p, layout, dtype=dtype, **kw)
            c.v[at] = v_new[row].double().numpy()
            want_q[x, :, i], err_q[x, :, i] = R.rotate(q[x, :, i].double().numpy(), np.full(g, p), layout, dtype=dtype, **kw)
    d.same(err)
    R.check(host(q_out), want_q, err_q, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_append_without_queries_or_with_them_in_place(grkv_lib, dtype):
    rng = np.random.default_rng(2)
    c = C.Cache([20, 77], 16, dtype, 3)
    a, d = Dev(c, 3, 6), Dev(c, 3, 6)
    k_new, v_new, q = (normal(rng, dtype, 2, *s, 6, D).cuda() for s in ((), (), (3,)))
    rope = plan()
    b.grkv_cache_append_rope(a.p, rope, k_new, v_new, a.k, a.v, a.table, a.lens, a.ws)
    out = torch.empty_like(q)
    b.grkv_rope_rows(rope, q, out, pos=(a.lens[:, None] - 6 + torch.arange(6, device="cuda")).int())
    b.grkv_cache_append_rope(d.p, rope, k_new, v_new, d.k, d.v, d.table, d.lens, d.ws, q=q, q_out=q)
    assert torch.equal(q, out)
    assert np.array_equal(host(a.k), host(d.k), equal_nan=True)
    # the keys are those of the rows' operator, bit for bit, appended
    keys, e = torch.empty_like(k_new), Dev(c, 3, 6)
    b.grkv_rope_rows(rope, k_new[:, None], keys[:, None], start=a.lens - 6)
    b.grkv_cache_append(e.p, keys, v_new, e.k, e.v, e.table, e.lens, e.ws)
    for x, y in ((e.k, a.k), (e.v, a.v)):
        assert np.array_equal(host(x), host(y), equal_nan=True)


def test_append_reports_rows_without_a_place(grkv_lib):
    """No page, behind the table, before the first slot, packed rows that are not there, positions below
    zero: those rows are left out and reported, the others go where they belong."""
    page, t, dtype = 16, 4, "f32"
    for fault in ("page", "long", "short", "row", "position", "offset", "none"):
        c = C.Cache([20, 40, 64], page, dtype, 5)
        u = 3
        lens, first, pos = list(c.lens), [0, 4, 8], np.arange(12) + 100
        offset = None
        if fault == "page":
            c.k[c.table[1, 2]] = c.v[c.table[1, 2]] = np.nan
            c.table[1, 2] = -1
        if fault == "long":
            lens[2] = 66
        if fault == "short":
            lens[0] = 2
        if fault == "row":
            first[2] = 10
        if fault == "position":
            pos[5] = -1
        if fault == "offset":
            offset, pos = [0, -38, 7], None
        d = Dev(c, 2, t)
        d.lens = C.int_dev(lens)
        rng = np.random.default_rng(6)
        k_new, v_new, q = normal(rng, dtype, 12, D), normal(rng, dtype, 12, D), normal(rng, dtype, u, 2, t, D)
        q_out = torch.full(q.shape, 7.0, dtype=torch.float32, device="cuda")
        b.grkv_cache_append_rope(
            d.p, plan(), k_new.cuda(), v_new.cuda(), d.k, d.v, d.table, d.lens, d.ws, q=q.cuda(), q_out=q_out,
            pos=None if pos is None else C.int_dev(pos), first_row=torch.tensor(first).cuda(),
            offset=None if offset is None else C.int_dev(offset))
        err, want, err_q = np.zeros_like(c.k), np.full(q.shape, 7.0), np.zeros(q.shape)
        for x in range(u):
            for i in range(t):
                slot, row = lens[x] - t + i, first[x] + i
                p = -1 if row > 11 else pos[row] if pos is not None else slot + offset[x]
                if p < 0:
                    continue
                want[x, :, i], err_q[x, :, i] = R.rotate(q[x, :, i].double().numpy(), np.full(2, p))
                if slot < 0 or slot >= c.cols * page or c.table[x, slot // page] < 0:
                    continue
                at = C.at(c.table, x, slot, page)
                c.k[at], err[at] = R.rotate(k_new[row].double().numpy(), p)
                c.v[at] = v_new[row].double().numpy()
        d.same(err, b.GRKV_OK if fault == "none" else b.GRKV_ERR_INVALID_ARG)
        R.check(host(q_out), want, err_q, dtype)


def test_append_reports_counts_outside_their_range(grkv_lib):
    c = C.Cache([20, 40], 16, "f32", 5)
    d = Dev(c, 1, 3)
    k_new, v_new = (normal(np.random.default_rng(6), "f32", 2, 3, D) for _ in range(2))
    b.grkv_cache_append_rope(d.p, plan(), k_new.cuda(), v_new.cuda(), d.k, d.v, d.table, d.lens, d.ws,
                             count=C.int_dev([-2, 9]))
    err = np.zeros_like(c.k)
    for i in range(3):                       # 9 counts as 3, -2 as none
        at = C.at(c.table, 1, 37 + i, 16)
        c.k[at], err[at] = R.rotate(k_new[1, i].double().numpy(), 37 + i)
        c.v[at] = v_new[1, i].double().numpy()
    d.same(err, b.GRKV_ERR_INVALID_ARG)


# ----------------------------------------------------------------------- compact
def kept(rng, n, m):
    return np.sort(rng.permutation(n)[:m])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout,rotary", [("half", 128), ("half", 96), ("half", 22), ("pairs", 128),
                                           ("pairs", 14)])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("place", ["other", "in place"])
@pytest.mark.parametrize("given", [False, True])
def test_compact(grkv_lib, dtype, layout, rotary, page, place, given):
    """Kept rows to other pages and in place, keys turned by their slots' change or a given number."""
    rng = np.random.default_rng(rotary + page)
    lens, keep, first = [700, 1200, 40, 5], [300, 640, 40, 0], [0, 17, 0, 2]
    t, u = 640, 4
    c = C.Cache(lens + ([700, 700, 700, 700] if place == "other" else []), page, dtype, 7)
    table_out = c.table[u:].copy() if place == "other" else c.table[:u]
    c.lens, c.table = c.lens[:u], c.table[:u].copy()
    d = Dev(c, 1, t)
    d.table = C.int_dev(c.table)
    idx, turn = np.full((u, t), 1 << 29, np.int32), rng.integers(-5000, 5000, (u, t))
    turn[:, ::3] = 0
    for x in range(u):
        idx[x, :keep[x]] = first[x] + kept(rng, lens[x] - first[x], keep[x])
    kw = dict(rotary=rotary, scaling="ntk", factor=2.0)
    to = d.table if place == "in place" else C.int_dev(table_out)
    b.grkv_cache_compact_rope(d.p, plan(layout, amplitude=3.0, **kw), C.int_dev(idx), d.k, d.v, d.table, d.lens,
                              to, d.ws, keep=C.int_dev(keep), first=C.int_dev(first),
                              turn=C.int_dev(turn) if given else None)
    before_k, before_v, err = c.k.copy(), c.v.copy(), np.zeros_like(c.k)
    exact = np.zeros(c.k.shape[:2], bool)
    for x in range(u):
        for i in range(keep[x]):
            src, dst = C.at(c.table, x, idx[x, i], page), C.at(table_out, x, first[x] + i, page)
            by = turn[x, i] if given else first[x] + i - idx[x, i]
            c.k[dst], err[dst] = R.rotate(before_k[src], by, layout, amplitude=1.0, dtype=dtype, **kw)
            if by == 0:
                c.k[dst], err[dst], exact[dst] = before_k[src], 0.0, True
            c.v[dst] = before_v[src]
    d.same(err)
    assert np.array_equal(host(d.k)[exact], c.k[exact])


@pytest.mark.parametrize("dtype", TYPES)
def test_keys_that_are_not_turned_move_as_they_are(grkv_lib, dtype):
    """NaN and infinities too, to the bit what grkv_cache_compact does."""
    rng = np.random.default_rng(9)
    for same in (False, True):
        c = C.Cache([500, 500], 32, dtype, 10)
        c.k[c.table[0, 3], 5, ::7], c.k[c.table[0, 4], 6, 3] = np.nan, np.inf
        out = c.table[0:1] if same else c.table[1:2]
        c.lens, c.table = [500], c.table[:1]
        a, d = Dev(c, 1, 333), Dev(c, 1, 333)
        idx = C.int_dev(kept(rng, 500, 333)[None])
        tb = a.table if same else C.int_dev(out)
        b.grkv_cache_compact(a.p, idx, a.k, a.v, a.table, a.lens, tb, a.ws)
        tb = d.table if same else C.int_dev(out)
        b.grkv_cache_compact_rope(d.p, plan(), idx, d.k, d.v, d.table, d.lens, tb, d.ws,
                                  turn=torch.zeros_like(idx))
        assert b.grkv_status(d.ws) == b.GRKV_OK
        word = torch.int16 if dtype == "bf16" else torch.int32
        assert torch.equal(a.k.view(word), d.k.view(word)) and torch.equal(a.v.view(word), d.v.view(word))


@pytest.mark.parametrize("same", [False, True])
def test_compact_reports_what_its_contract_excludes(grkv_lib, same):
    c = C.Cache([100, 100], 16, "f32", 11)
    out = c.table[0:1].copy() if same else c.table[1:2].copy()
    c.lens, c.table = [100], c.table[:1]
    d = Dev(c, 1, 6)
    idx = [3, 100, -1, 20, 1 << 30, 50] if not same else [3, 100, -1, 20, 2, 50]
    tb = d.table if same else C.int_dev(out)
    b.grkv_cache_compact_rope(d.p, plan(), C.int_dev([idx]), d.k, d.v, d.table, d.lens, tb, d.ws)
    before, bv, err = c.k.copy(), c.v.copy(), np.zeros_like(c.k)
    for i in (0, 3, 5):
        src, dst = C.at(c.table, 0, idx[i], 16), C.at(out, 0, i, 16)
        c.k[dst], err[dst] = R.rotate(before[src], i - idx[i])
        c.v[dst] = bv[src]
    d.same(err, b.GRKV_ERR_INVALID_ARG)


def test_turned_keys_are_those_of_their_new_positions(grkv_lib):
    """Appended at their slots, compacted in place: logits with a query depend on slots alone."""
    rng = np.random.default_rng(12)
    n, m = 300, 120
    c = C.Cache([n], 16, "f32", 13)
    d = Dev(c, 1, n)
    rope = plan("pairs", rotary=64, scaling="yarn", factor=4.0)
    k_new, v_new = normal(rng, "f32", 1, n, D).cuda(), normal(rng, "f32", 1, n, D).cuda()
    b.grkv_cache_append_rope(d.p, rope, k_new, v_new, d.k, d.v, d.table, d.lens, d.ws)
    idx = kept(rng, n, m)
    p = b.cache_params(1, 1, c.pages, 16, c.cols, tokens=m, dtype="f32")
    b.grkv_cache_compact_rope(p, rope, C.int_dev(idx[None]), d.k, d.v, d.table, d.lens, d.table, d.ws)
    want, err = R.rotate(host(k_new)[0, idx], np.arange(m), "pairs", rotary=64, scaling="yarn", factor=4.0)
    got = host(d.k)[c.table[0]].reshape(-1, D)[:m]
    # rounded in between: half a step, and the second turn's own errors
    R.check(got, want, 2.2 * err + 2.0 ** -23 * np.abs(want) + 2.0 ** -22, "f32")


@pytest.mark.parametrize("u", [0, 1, 70000])
def test_numbers_of_units(grkv_lib, u):
    """None, one, and more than a grid's second dimension holds."""
    page, g = 16, 1
    pages = max(1, 2 * u)
    p = b.cache_params(u, g, pages, page, 1)
    k = torch.zeros(pages, page, D, dtype=torch.bfloat16, device="cuda")
    v, rope = torch.zeros_like(k), plan()
    k_new = torch.randn(u, 1, D, dtype=torch.float32, device="cuda").bfloat16()
    table = torch.arange(u, dtype=torch.int32, device="cuda")
    lens = torch.full((u,), 9, dtype=torch.int32, device="cuda")
    ws = torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")
    b.grkv_cache_append_rope(p, rope, k_new, k_new, k, v, table, lens, ws, q=k_new, q_out=k_new.clone())
    assert b.grkv_status(ws) == b.GRKV_OK
    want = torch.empty(u, 1, 1, D, dtype=torch.bfloat16, device="cuda")
    if u:
        b.grkv_rope_rows(rope, k_new[:, None], want, start=lens - 1)
    assert torch.equal(k[:u, 8], want[:, 0, 0]) and torch.equal(v[:u, 8], k_new[:, 0])
    assert int((k[:u] != 0).any(-1).sum()) == u
    idx = torch.full((u, 1), 8, dtype=torch.int32, device="cuda")
    b.grkv_cache_compact_rope(p, rope, idx, k, v, table, lens, table + u, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
    if u:
        b.grkv_rope_rows(rope, k_new[:, None], want, start=torch.zeros_like(lens))
        assert (k[u:, 0].float() - want[:, 0, 0].float()).abs().max() < 0.1
        assert torch.equal(v[u:, 0], k_new[:, 0])
