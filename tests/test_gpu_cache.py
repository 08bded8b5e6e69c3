"""The paged cache's page operators against plain bookkeeping, and a run of them together with
the attention, as a serving loop uses them after grkv_compress."""
import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
D = R.D


class Dev:
    """A cache on the device beside its copy in numpy."""

    def __init__(self, c, tokens=1, **kw):
        self.c = c
        self.p = b.cache_params(len(c.lens), 2, c.pages, c.page, c.cols, tokens=tokens,
                                dtype=c.dtype, **kw)
        self.k, self.v = c.dev()
        self.table, self.lens, self.refs = (R.int_dev(x) for x in (c.table, c.lens, c.refs))
        self.ws = torch.full((b.grkv_cache_workspace_size(self.p),), 0xFF, dtype=torch.uint8,
                             device="cuda")

    def ok(self, code=b.GRKV_OK):
        assert b.grkv_status(self.ws) == code

    def same(self):
        c = self.c
        assert np.array_equal(self.table.cpu().numpy(), c.table)
        assert np.array_equal(self.refs.cpu().numpy(), c.refs)
        for got, want in ((self.k, c.k), (self.v, c.v)):
            assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


TYPES = ["bf16", "f32"]
LENS = [1, 15, 16, 17, 64, 100, 0, 333, 128]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [16, 64, 128])
def test_reserve_takes_the_lowest_free_pages(grkv_lib, dtype, page):
    c = R.Cache(LENS, page, dtype, 1, spare=60, extra_cols=4)
    want = [x + y for x, y in zip(LENS, [0, 1, 1, 15, 3 * page, 1, page, -5, 0])]
    d = Dev(c)
    b.grkv_cache_reserve(d.p, d.table, d.lens, R.int_dev(want), d.refs, d.k, d.v, d.ws)
    d.ok()
    assert R.reserve(c.table, c.lens, want, c.refs, c.k, c.v, page)
    d.same()


@pytest.mark.parametrize("dtype", TYPES)
def test_reserve_copies_shared_pages(grkv_lib, dtype):
    """Three forks of each unit write behind a shared, partly filled page."""
    page = 32
    c = R.Cache([10, 32, 70, 95, 0], page, dtype, 2, spare=80, extra_cols=2)
    src = [0, 0, 0, 1, 1, 2, 2, 2, 3, 4, 4, -1]
    d = Dev(c)
    pf = b.cache_params(len(src), 2, c.pages, page, c.cols, dtype=dtype)
    table = torch.full((len(src), c.cols), 99, dtype=torch.int32, device="cuda")
    lens = torch.full((len(src),), 99, dtype=torch.int32, device="cuda")
    b.grkv_cache_fork(pf, R.int_dev(src), d.table, d.lens, table, lens, d.refs, d.ws)
    d.ok()
    t2, l2 = R.fork(src, c.table, c.lens, c.refs, c.cols, page)
    assert np.array_equal(table.cpu().numpy(), t2) and np.array_equal(lens.cpu().numpy(), l2)
    d.same()
    # the parents go; what is left has counts of 1 to 3
    none = torch.zeros_like(d.lens)
    b.grkv_cache_trim(d.p, d.table, none, d.refs, d.ws)
    d.ok()
    R.trim(c.table, [0] * 5, c.refs, page)
    d.same()
    want = [int(x) + 1 + i % 3 for i, x in enumerate(l2)]
    b.grkv_cache_reserve(pf, table, lens, R.int_dev(want), d.refs, d.k, d.v, d.ws)
    d.ok()
    assert R.reserve(t2, l2, want, c.refs, c.k, c.v, page)
    assert np.array_equal(table.cpu().numpy(), t2)
    d.same()


def test_reserve_of_many_units_and_pages(grkv_lib):
    """More units than threads of the block, more pages than one sweep looks at."""
    rng = np.random.default_rng(3)
    units, page, pages, cols = 2500, 16, 40000, 12
    lens = rng.integers(0, 100, units)
    need = np.array([R.pages_of(int(n), page) for n in lens])
    order = rng.permutation(pages)
    table = np.full((units, cols), -1, np.int32)
    at = 0
    for u in range(units):
        table[u, :need[u]] = order[at:at + need[u]]
        at += need[u]
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    refs[: pages // 2] += refs[: pages // 2] == 0        # held by another table
    want = lens + rng.integers(0, 80, units)
    k = np.zeros((pages, page, 1))
    p = b.cache_params(units, 1, pages, page, cols)
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    dk, dv = (torch.zeros(pages, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dt, dr = R.int_dev(table), R.int_dev(refs)
    b.grkv_cache_reserve(p, dt, R.int_dev(lens), R.int_dev(want), dr, dk, dv, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
    assert R.reserve(table, lens, want, refs, k, k.copy(), page)
    assert np.array_equal(dt.cpu().numpy(), table) and np.array_equal(dr.cpu().numpy(), refs)


def test_reserve_without_enough_pages_changes_nothing(grkv_lib):
    c = R.Cache([100, 100], 16, "bf16", 4, spare=3, extra_cols=6)
    d = Dev(c)
    b.grkv_cache_reserve(d.p, d.table, d.lens, R.int_dev([140, 130]), d.refs, d.k, d.v, d.ws)
    d.ok(b.GRKV_ERR_NO_PAGES)
    d.same()
    b.grkv_cache_reserve(d.p, d.table, d.lens, R.int_dev([140, 112]), d.refs, d.k, d.v, d.ws)
    d.ok()
    assert R.reserve(c.table, c.lens, [140, 112], c.refs, c.k, c.v, 16)
    d.same()


def test_trim(grkv_lib):
    c = R.Cache(LENS, 16, "bf16", 5)
    d = Dev(c)
    keep = [0, 15, 0, 16, 33, 100, 0, 1, 127]
    b.grkv_cache_trim(d.p, d.table, R.int_dev(keep), d.refs, d.ws)
    d.ok()
    R.trim(c.table, keep, c.refs, 16)
    d.same()


@pytest.mark.parametrize("dtype", TYPES)
def test_append(grkv_lib, dtype):
    t = 40
    c = R.Cache(LENS, 16, dtype, 6)
    count = [1, 0, 16, 17, 40, 3, 0, 40, 40]
    rng = np.random.default_rng(7)
    kn, vn = (c.rounded(rng.standard_normal((len(LENS), t, D))) for _ in range(2))
    d = Dev(c, tokens=t)
    as_t = lambda x: torch.from_numpy(x).to(R.TORCH[dtype]).cuda()
    b.grkv_cache_append(d.p, as_t(kn), as_t(vn), d.k, d.v, d.table, d.lens, d.ws,
                        count=R.int_dev(count))
    d.ok()
    for u, n in enumerate(LENS):
        for i in range(count[u]):
            at = R.at(c.table, u, n - count[u] + i, 16)
            c.k[at], c.v[at] = kn[u, i], vn[u, i]
    d.same()


def test_append_of_packed_rows(grkv_lib):
    """The outputs of a ragged compression: unit u's rows follow those of the units before."""
    c = R.Cache(LENS, 64, "bf16", 8)
    rng = np.random.default_rng(9)
    first = np.concatenate([[0], np.cumsum(LENS)])
    kn, vn = (c.rounded(rng.standard_normal((first[-1], D))) for _ in range(2))
    d = Dev(c, tokens=max(LENS))
    as_t = lambda x: torch.from_numpy(x).bfloat16().cuda()
    b.grkv_cache_append(d.p, as_t(kn), as_t(vn), d.k, d.v, d.table, d.lens, d.ws, count=d.lens,
                        first_row=torch.from_numpy(first[:-1].astype(np.int64)).cuda())
    d.ok()
    for u, n in enumerate(LENS):
        for i in range(n):
            at = R.at(c.table, u, i, 64)
            c.k[at], c.v[at] = kn[first[u] + i], vn[first[u] + i]
    d.same()


def kept(lens, keep, seed, lo=0):
    rng = np.random.default_rng(seed)
    return [sorted(rng.choice(np.arange(lo, n), k, replace=False)) for n, k in zip(lens, keep)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page", [16, 128])
def test_compact(grkv_lib, dtype, in_place, page):
    lens = [1, 15, 700, 300, 64, 1500, 0]
    keep = [1, 7, 700, 20, 63, 1200, 0]
    c = R.Cache(lens, page, dtype, 10, spare=R.pages_of(1200, page) * 7 + 5)
    d = Dev(c, tokens=1200)
    chosen = kept(lens, keep, 11)
    idx = np.zeros((7, 1200), np.int32)
    for u, x in enumerate(chosen):
        idx[u, :keep[u]] = x
    to = c.table
    if not in_place:
        free = [p for p in range(c.pages) if c.refs[p] == 0]
        to = np.full_like(c.table, -1)
        for u in range(7):
            for col in range(R.pages_of(keep[u], page)):
                to[u, col] = free.pop()
    d_to = d.table if in_place else R.int_dev(to)
    b.grkv_cache_compact(d.p, R.int_dev(idx), d.k, d.v, d.table, d.lens, d_to, d.ws,
                         keep=R.int_dev(keep))
    d.ok()
    for u in range(7):
        k, v = c.slots(u)
        k, v = k.copy(), v.copy()
        for i, j in enumerate(chosen[u]):
            at = R.at(to, u, i, page)
            c.k[at], c.v[at] = k[j], v[j]
    d.same()
    if in_place:      # the rest of the pages goes back
        b.grkv_cache_trim(d.p, d.table, R.int_dev(keep), d.refs, d.ws)
        d.ok()
        R.trim(c.table, keep, c.refs, page)
        d.same()


def test_compact_of_an_accepted_path(grkv_lib):
    """Slots before `first` stay; the same slot may be kept twice where it lies far enough."""
    lens, first, page = [100, 40, 64], [90, 20, 64], 16
    idx = np.array([[91, 93, 99, 0], [20, 21, 39, 39], [0, 0, 0, 0]], np.int32)
    keep = [3, 4, 0]
    c = R.Cache(lens, page, "bf16", 12)
    d = Dev(c, tokens=4)
    b.grkv_cache_compact(d.p, R.int_dev(idx), d.k, d.v, d.table, d.lens, d.table, d.ws,
                         keep=R.int_dev(keep), first=R.int_dev(first))
    d.ok()
    for u in range(3):
        k, v = (x.copy() for x in c.slots(u))
        for i in range(keep[u]):
            at = R.at(c.table, u, first[u] + i, page)
            c.k[at], c.v[at] = k[idx[u, i]], v[idx[u, i]]
    d.same()


def test_faults_are_reported_and_nothing_else_moves(grkv_lib):
    page = 16
    inv = b.GRKV_ERR_INVALID_ARG
    new = lambda: Dev(R.Cache([40, 20], page, "bf16", 13, spare=9, extra_cols=1), tokens=2)
    rows = torch.ones(2, 2, D, dtype=torch.bfloat16, device="cuda")
    big = 2 ** 31 - 1
    # append: no page, a bad entry, a count or a length out of range, slots before the first
    for col, entry in ((1, -1), (1, big), (1, -2 ** 31)):
        d = new()
        d.table[1, col] = entry
        d.c.table[1, col] = entry
        b.grkv_cache_append(d.p, rows[:, :2], rows, d.k, d.v, d.table, d.lens, d.ws,
                            count=R.int_dev([0, 2]))
        d.ok(inv)
        d.same()
    for lens, count in (([1, 20], [2, 0]), ([40, 20], [-1, 0]), ([-7, 20], [0, 0]),
                        ([big, 20], [0, 0])):
        d = new()
        if lens == [1, 20]:
            d.c.k[d.c.table[0, 0], 0] = d.c.v[d.c.table[0, 0], 0] = 1
        b.grkv_cache_append(d.p, rows, rows, d.k, d.v, d.table, R.int_dev(lens), d.ws,
                            count=R.int_dev(count))
        d.ok(inv)
        d.same()
    # append of packed rows that are not there
    for first in (-1, 3, 2 ** 62, -2 ** 63):
        d = new()
        b.grkv_cache_append(d.p, rows, rows, d.k, d.v, d.table, d.lens, d.ws,
                            count=R.int_dev([2, 0]),
                            first_row=torch.tensor([first, 0], dtype=torch.int64, device="cuda"))
        d.ok(inv)
        if first == 3:                          # the first of two rows is the last there is
            at = R.at(d.c.table, 0, 38, page)
            d.c.k[at] = d.c.v[at] = 1
        d.same()
    # compact: sources out of range, or before their place
    for idx, first in (([[40, 0]], 0), ([[-1, 0]], 0), ([[4, 5]], 30), ([[5, 6]], -1),
                       ([[5, 6]], big)):
        d = new()
        b.grkv_cache_compact(d.p, R.int_dev(idx * 2), d.k, d.v, d.table, d.lens, d.table, d.ws,
                             keep=R.int_dev([1, 0]), first=R.int_dev([first, 0]))
        d.ok(inv)
        d.same()
    # fork: a parent that is not there
    for s in (2, -2, big):
        d = new()
        t2, l2 = torch.zeros_like(d.table), torch.zeros_like(d.lens)
        b.grkv_cache_fork(d.p, R.int_dev([s, -1]), d.table, d.lens, t2, l2, d.refs, d.ws)
        d.ok(inv)
        assert (t2 == -1).all() and (l2 == 0).all()
        d.same()
    # trim: a page that nobody holds, an entry out of range
    d = new()
    free = int(np.flatnonzero(d.c.refs == 0)[0])
    d.table[0, 3], d.table[1, 3] = free, big
    d.c.table[0, 3] = d.c.table[1, 3] = -1
    b.grkv_cache_trim(d.p, d.table, d.lens, d.refs, d.ws)
    d.ok(inv)
    d.same()
    # reserve: more than the table holds
    d = new()
    b.grkv_cache_reserve(d.p, d.table, d.lens, R.int_dev([big, 20]), d.refs, d.k, d.v, d.ws)
    d.ok(inv)
    R.reserve(d.c.table, d.c.lens, [d.c.cols * page, 20], d.c.refs, d.c.k, d.c.v, page)
    d.same()


def test_compressed_caches_are_decoded_with_drafts(grkv_lib):
    """grkv_compress_ragged, its outputs into pages, a decoding step, a drafted tree, the
    accepted path, the next step: every attention against the formula on the rows it should see."""
    units, g, n, w, page = 6, 4, 900, 16, 32
    budgets = [100, 64, 333, 64, 17, 250]
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float32, device="cuda", generator=gen).bfloat16()
    q, k, v = rnd(units, g, w, D), rnd(units, n, D), rnd(units, n, D)
    p = b.params(units, g, n, w, max(budgets))
    rows = sum(budgets)
    ko, vo = rnd(rows, D), rnd(rows, D)
    idx = torch.empty(rows, dtype=torch.int32, device="cuda")
    cws = torch.empty(b.grkv_compress_ragged_workspace_size(p, budgets), dtype=torch.uint8,
                      device="cuda")
    b.grkv_compress_ragged(p, budgets, q, k, v, ko, vo, idx, cws)
    assert b.grkv_status(cws) == b.GRKV_OK
    pages, cols, t = 60, 14, 9
    pool = [torch.full((pages, page, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            for _ in range(2)]
    table = torch.full((units, cols), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    lens = torch.zeros(units, dtype=torch.int32, device="cuda")
    cp = lambda tokens, **kw: b.cache_params(units, g, pages, page, cols, tokens=tokens, **kw)
    ws = torch.empty(b.grkv_cache_workspace_size(cp(max(budgets))), dtype=torch.uint8, device="cuda")
    ok = lambda: b.grkv_status(ws)
    first = np.concatenate([[0], np.cumsum(budgets)[:-1]])
    hist = [(ko[f:f + m].double().cpu().numpy(), vo[f:f + m].double().cpu().numpy())
            for f, m in zip(first, budgets)]

    def grow(rows_per_unit, kn, vn, **kw):
        nonlocal lens
        count = torch.tensor(rows_per_unit, dtype=torch.int32, device="cuda")
        want = lens + count
        tok = cp(max(rows_per_unit))
        b.grkv_cache_reserve(tok, table, lens, want, refs, *pool, ws)
        assert ok() == b.GRKV_OK
        b.grkv_cache_append(tok, kn, vn, *pool, table, want, ws, count=count, **kw)
        assert ok() == b.GRKV_OK
        lens = want

    def attend(tokens, parents=None, window=0):
        qq = rnd(units, g, tokens, D) * 1.5
        out = torch.empty_like(qq)
        pa = cp(tokens, window=window)
        if parents is None:
            b.grkv_attend(pa, qq, *pool, table, lens, out, ws)
        else:
            b.grkv_attend_tree(pa, qq, *pool, table, lens, R.int_dev(parents), out, ws)
        assert ok() == b.GRKV_OK
        for u in range(units):
            par = None if parents is None else parents[u]
            o, _, mass, err = R.attend_unit(qq[u].double().cpu().numpy(), *hist[u], tokens, window,
                                            4, None, par)
            tol = (2 * err + 2.0 ** -13 + 2.0 ** -8)[..., None] * mass + 2.0 ** -8 * np.abs(o)
            assert (np.abs(out[u].double().cpu().numpy() - o) <= tol).all()

    def add(kn, vn):
        for u in range(units):
            hist[u] = (np.concatenate([hist[u][0], kn[u].double().cpu().numpy()]),
                       np.concatenate([hist[u][1], vn[u].double().cpu().numpy()]))

    grow(budgets, ko, vo, first_row=torch.tensor(first, dtype=torch.int64, device="cuda"))
    for step in range(2):
        kn, vn = rnd(units, 1, D), rnd(units, 1, D)
        grow([1] * units, kn, vn)
        add(kn, vn)
        attend(1)
        attend(1, window=50)
    base, before = lens.clone(), list(hist)
    kn, vn = rnd(units, t, D), rnd(units, t, D)
    grow([t] * units, kn, vn)
    add(kn, vn)
    parents = [[-1, 0, 0, 1, 1, 2, -1, 6, 3]] * units
    attend(t, parents)
    paths = [[0, 1, 3, 8], [0, 2, 5], [6, 7], [6], [0, 1, 4], []]
    idx2 = np.zeros((units, t), np.int32)
    for u, path in enumerate(paths):
        idx2[u, :len(path)] = [int(base[u]) + x for x in path]
        hist[u] = tuple(np.concatenate([before[u][s], x[u].double().cpu().numpy()[path]])
                        for s, x in ((0, kn), (1, vn)))
    keep = R.int_dev([len(x) for x in paths])
    b.grkv_cache_compact(cp(t), R.int_dev(idx2), *pool, table, lens, table, ws, keep=keep, first=base)
    assert ok() == b.GRKV_OK
    lens = base + keep
    b.grkv_cache_trim(cp(1), table, lens, refs, ws)
    assert ok() == b.GRKV_OK
    attend(1)
    kn, vn = rnd(units, 3, D), rnd(units, 3, D)
    grow([3] * units, kn, vn)
    add(kn, vn)
    attend(3)
    held = (table >= 0).sum().item()
    assert refs.sum().item() == held == sum(R.pages_of(int(x), page) for x in lens.tolist())


def test_no_units(grkv_lib):
    p = b.cache_params(0, 1, 8, 16, 4)
    ws = torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    rows = torch.empty(0, dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros(8, 16, D, dtype=torch.bfloat16, device="cuda")
    refs = torch.zeros(8, dtype=torch.int32, device="cuda")
    for call in (lambda: b.grkv_cache_trim(p, e, e, refs, ws),
                 lambda: b.grkv_cache_reserve(p, e, e, e, refs, pool, pool, ws),
                 lambda: b.grkv_cache_append(p, rows, rows, pool, pool, e, e, ws),
                 lambda: b.grkv_cache_compact(p, e, pool, pool, e, e, e, ws),
                 lambda: b.grkv_cache_fork(p, e, e, e, torch.empty_like(e), torch.empty_like(e),
                                           refs, ws)):
        ws[:4] = 0xFF
        call()
        assert b.grkv_status(ws) == b.GRKV_OK


@pytest.mark.parametrize("units,cols", [(7, 5), (300, 40)])
def test_fork_and_trim_of_small_and_large_tables(grkv_lib, units, cols):
    """One block that writes the status itself, and many that add to a cleared word."""
    rng = np.random.default_rng(units)
    page = 16
    c = R.Cache([int(x) for x in rng.integers(0, (cols - 1) * page, units)], page, "bf16", 3)
    c.table = np.concatenate([c.table, np.full((units, cols - c.cols), -1, np.int32)], 1)
    c.cols = cols
    d = Dev(c)
    src = [int(x) for x in rng.integers(-1, units, units)]
    t2, l2 = R.fork(src, c.table, c.lens, c.refs, cols, page)
    table, lens = torch.full_like(d.table, 5), torch.full_like(d.lens, 5)
    b.grkv_cache_fork(d.p, R.int_dev(src), d.table, d.lens, table, lens, d.refs, d.ws)
    d.ok()
    assert np.array_equal(table.cpu().numpy(), t2) and np.array_equal(lens.cpu().numpy(), l2)
    d.same()
    half = [int(x) // 2 for x in l2]
    b.grkv_cache_trim(d.p, table, R.int_dev(half), d.refs, d.ws)
    d.ok()
    R.trim(t2, half, c.refs, page)
    assert np.array_equal(table.cpu().numpy(), t2)
    d.same()
    bad = R.int_dev([units] + src[1:])
    table.fill_(-1)
    b.grkv_cache_fork(d.p, bad, d.table, d.lens, table, lens, d.refs, d.ws)
    d.ok(b.GRKV_ERR_INVALID_ARG)
    b.grkv_cache_trim(d.p, table, torch.zeros_like(lens), d.refs, d.ws)
    d.ok()


def test_pools_beyond_32_bit_offsets(grkv_lib):
    """Pages whose elements lie past 2^31: every call that reads or writes them."""
    pages, page, n, t = 140000, 128, 300, 3         # 2.3e9 elements a pool
    pool = [torch.empty(pages, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far = [139999, 7, 139000, 138000]
    table = R.int_dev([far])
    lens, refs = R.int_dev([n]), torch.ones(pages, dtype=torch.int32, device="cuda")
    p = b.cache_params(1, 2, pages, page, 4, tokens=n)
    ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float32, device="cuda", generator=gen).bfloat16()
    kn, vn = rnd(1, n, D), rnd(1, n, D)
    b.grkv_cache_append(p, kn, vn, *pool, table, lens, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
    got = torch.cat([pool[0][x] for x in far[:3]])[:n]
    assert torch.equal(got, kn[0])
    for flags in (0, b.GRKV_FORCE_SIMT):
        pq = b.cache_params(1, 2, pages, page, 4, tokens=t, flags=flags)
        q, out = rnd(1, 2, t, D), rnd(1, 2, t, D)
        b.grkv_attend(pq, q, *pool, table, lens, out, ws)
        assert b.grkv_status(ws) == b.GRKV_OK
        o, _, mass, err = R.attend_unit(q[0].double().cpu().numpy(), kn[0].double().cpu().numpy(),
                                        vn[0].double().cpu().numpy(), t, 0, 4)
        tol = (2 * err + 2.0 ** -13 + 2.0 ** -8)[..., None] * mass + 2.0 ** -8 * np.abs(o)
        assert (np.abs(out[0].double().cpu().numpy() - o) <= tol).all()
    pc = b.cache_params(1, 2, pages, page, 4, tokens=2)
    b.grkv_cache_compact(pc, R.int_dev([[5, 299]]), *pool, table, lens, table, ws,
                         first=R.int_dev([2]))
    assert b.grkv_status(ws) == b.GRKV_OK
    assert torch.equal(pool[1][far[0], 2:4], vn[0, [5, 299]])
    refs[:139998] = 2                               # two free pages, at the end
    refs[139998:] = 0
    b.grkv_cache_reserve(pc, table, R.int_dev([130]), R.int_dev([140]), refs, *pool, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
    assert table[0, 1].item() == 139998
    assert torch.equal(pool[0][139998, :2], kn[0, 128:130])
