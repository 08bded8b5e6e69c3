"""grkv_attend and grkv_attend_tree against their formulas in 64 bits.  Every slot that is not
part of a unit is NaN, and so is every page that no unit holds."""
import math

import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
D = R.D


def workspace(p):
    return torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")


def queries(u, g, t, dtype, seed, std=1.5):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((u, g, t, D)) * std).to(R.TORCH[dtype])
    return x, x.double().numpy()


def check(c, p, q64, out, lse, q_lens, parents=None, scale=None, tensor_cores=False):
    window, sink, t = p.window, p.n_sink, p.tokens
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for u in range(p.units):
        k, v = c.slots(u)
        par = None if parents is None else list(parents[u][:q_lens[u]])
        o, z, mass, err = R.attend_unit(q64[u], k, v, q_lens[u], window, sink, scale, par)
        n = len(k)
        rel = 2 * err + (n + 64) * R.U32 + 2.0 ** -21
        live = np.arange(t) < q_lens[u]
        tol = (rel + (2.0 ** -8 if c.dtype == "bf16" else 0))[..., None] * mass \
            + R.ROUND[c.dtype] * np.abs(o)
        bad = np.isnan(o)
        assert np.array_equal(np.isnan(got[u][:, live]), bad[:, live]), f"unit {u}: NaN rows"
        inf = np.isinf(o)
        assert np.array_equal(got[u][:, live][inf[:, live]], o[:, live][inf[:, live]])
        fine = ~bad & ~inf
        diff = np.abs(np.where(fine, got[u], 0) - np.where(fine, o, 0))
        over = (diff > np.where(fine, tol, 1))[:, live]
        assert not over.any(), (f"unit {u}: {over.sum()} off, worst "
                                f"{(diff / np.maximum(tol, 1e-30))[:, live].max():.2f} of the bound")
        empty = np.isneginf(z)
        gl = got_lse[u]
        assert np.array_equal(np.isneginf(gl[:, live]), empty[:, live])
        ok = np.isfinite(z) & live[None]
        assert (np.abs(gl[ok] - z[ok]) <= (rel + 4 * R.U32 * np.abs(z))[ok]).all()
        assert (got[u][:, ~live] == 7).all() and (gl[:, ~live] == 7).all(), "rows behind the last"


def run(c, p, q, q_lens=None, parents=None, stream=None):
    kd, vd = c.dev()
    out = torch.full(q.shape, 7, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:3], 7, dtype=torch.float32, device="cuda")
    ws = workspace(p)
    ql = None if q_lens is None else R.int_dev(q_lens)
    args = (kd, vd, R.int_dev(c.table), R.int_dev(c.lens))
    torch.cuda.synchronize()
    if parents is None:
        b.grkv_attend(p, q.cuda(), *args, out, ws, q_lens=ql, lse=lse, stream=stream)
    else:
        b.grkv_attend_tree(p, q.cuda(), *args, R.int_dev(parents), out, ws, q_lens=ql, lse=lse,
                           stream=stream)
    assert b.grkv_status(ws, stream) == b.GRKV_OK
    return out, lse


def attend_case(lens, g, t, page, dtype, window=0, sink=4, q_lens=None, flags=0, seed=0,
                parents=None, scale=0.0):
    c = R.Cache(lens, page, dtype, seed)
    q, q64 = queries(len(lens), g, t, dtype, seed + 1)
    p = b.cache_params(len(lens), g, c.pages, page, c.cols, tokens=t, window=window, n_sink=sink,
                       dtype=dtype, flags=flags, scale=scale)
    out, lse = run(c, p, q, q_lens, parents)
    check(c, p, q64, out, lse, q_lens or [t] * len(lens), parents, scale or None)
    return c, p, q, q64


TYPES = [("f32", 0), ("bf16", 0), ("bf16", b.GRKV_FORCE_SIMT)]


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decode_lengths(grkv_lib, dtype, flags, page):
    attend_case([1, 2, page - 1, page, page + 1, 127, 128, 129, 257, 1003, 0, 640], 4, 1, page,
                dtype, flags=flags)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g", [1, 3, 8, 64])
def test_decode_groups(grkv_lib, dtype, flags, g):
    attend_case([300, 5, 0, 1], g, 1, 16, dtype, flags=flags, seed=3)


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_one_long_unit_is_split_over_the_ctas(grkv_lib, dtype, flags):
    attend_case([30011], 2, 1, 64, dtype, flags=flags, seed=4)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 4), (100, 4), (128, 0), (300, 130), (5000, 2)])
@pytest.mark.parametrize("t", [1, 7, 150])
def test_window_and_sinks(grkv_lib, dtype, flags, window, sink, t):
    attend_case([900, 700, 151, 1, 0], 3, t, 32, dtype, window=window, sink=sink, flags=flags,
                seed=5, q_lens=[t, min(t, 3), t, 0, t])


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(1, 513), (4, 130), (7, 41), (64, 5), (5, 300)])
def test_chunks(grkv_lib, dtype, flags, g, t):
    """More queries than slots leave rows in front of the cache, which see nothing."""
    attend_case([t, t + 333, max(0, t - 40), 2 * t + 1], g, t, 16, dtype, flags=flags, seed=6)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("seed", range(4))
def test_random_shapes(grkv_lib, dtype, flags, seed):
    rng = np.random.default_rng(900 + seed)
    for k in range(4):
        u, g = int(rng.integers(1, 6)), int(rng.integers(1, 17))
        t = int(rng.integers(1, 2400 // (u * g) + 2))
        lens = [int(x) for x in rng.integers(0, 700, u)]
        attend_case(lens, g, t, int(rng.choice([16, 32, 64, 128])), dtype,
                    window=int(rng.choice([0, rng.integers(1, 400)])),
                    sink=int(rng.integers(0, 150)), flags=flags, seed=1000 * seed + k,
                    q_lens=[int(x) for x in rng.integers(0, t + 1, u)])


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_scale(grkv_lib, dtype, flags):
    attend_case([200, 90], 2, 3, 16, dtype, flags=flags, seed=8, scale=0.25)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_values_that_a_row_does_not_see_stay_out_of_it(grkv_lib, dtype, flags, what):
    """A NaN or an infinity in a value reaches the rows that see its slot and no other."""
    t, n = 200, 611
    for slot, window, sink in ((n - 1, 0, 0), (n - 77, 0, 0), (n - t - 50, 100, 4), (2, 100, 4),
                               (n - t, 64, 0)):
        c = R.Cache([n, 300], 32, dtype, 9)
        c.v[c.table[0, slot // 32], slot % 32, 5:9] = what
        q, q64 = queries(2, 2, t, dtype, 10)
        p = b.cache_params(2, 2, c.pages, 32, c.cols, tokens=t, window=window, n_sink=sink,
                           dtype=dtype, flags=flags)
        out, lse = run(c, p, q)
        check(c, p, q64, out, lse, [t, t])


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_keys_that_a_row_does_not_see_stay_out_of_it(grkv_lib, dtype, flags):
    t, n = 140, 400
    for what in (math.nan, math.inf):
        c = R.Cache([n], 16, dtype, 11)
        slot = n - 60
        c.k[c.table[0, slot // 16], slot % 16] = what
        q, q64 = queries(1, 1, t, dtype, 12)
        p = b.cache_params(1, 1, c.pages, 16, c.cols, tokens=t, dtype=dtype, flags=flags)
        out, lse = run(c, p, q)
        o = out.double().cpu().numpy()[0, 0]
        sees = np.arange(t) + n - t >= slot
        ref = R.attend_unit(q64[0], *c.slots(0), t, 0, 4)[0][0]
        assert np.isfinite(o[~sees]).all() and np.allclose(o[~sees], ref[~sees], atol=0.02)
        if math.isnan(what):
            assert np.isnan(o[sees]).all()


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_pages_out_of_every_window_may_be_gone(grkv_lib, dtype, flags):
    n, page, t, window, sink = 1000, 16, 5, 90, 20
    c = R.Cache([n], page, dtype, 13)
    for col in range(c.cols):
        lo, hi = col * page, (col + 1) * page
        if lo >= sink and hi <= n - t - window + 1:
            c.k[c.table[0, col]] = c.v[c.table[0, col]] = np.nan
            c.table[0, col] = -1
    q, q64 = queries(1, 4, t, dtype, 14)
    p = b.cache_params(1, 4, c.pages, page, c.cols, tokens=t, window=window, n_sink=sink,
                       dtype=dtype, flags=flags)
    out, lse = run(c, p, q)
    check(c, p, q64, out, lse, [t])


def trees(u, t, seed, back=6):
    rng = np.random.default_rng(seed)
    return [[max(-1, i - int(rng.integers(1, back + 1))) for i in range(t)] for _ in range(u)]


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(1, 1), (4, 13), (5, 64), (2, 256), (8, 33)])
@pytest.mark.parametrize("window", [0, 40])
def test_trees(grkv_lib, dtype, flags, g, t, window):
    par = trees(4, t, 15)
    par[1] = [i - 1 for i in range(t)]        # a chain
    par[2] = [-1] * t                         # every node a root
    attend_case([t + 500, t + 7, t, t + 129], g, t, 32, dtype, window=window, flags=flags,
                seed=16, parents=par, q_lens=[t, t, t, max(0, t - 2)])


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_a_chain_is_a_chunk(grkv_lib, dtype, flags):
    c = R.Cache([700, 333], 16, dtype, 17)
    q, _ = queries(2, 4, 30, dtype, 18)
    p = b.cache_params(2, 4, c.pages, 16, c.cols, tokens=30, window=77, dtype=dtype, flags=flags)
    o1, l1 = run(c, p, q)
    o2, l2 = run(c, p, q, parents=[[i - 1 for i in range(30)]] * 2)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_tree_nodes_do_not_see_values_of_other_branches(grkv_lib, dtype, flags):
    t, n = 40, 300
    par = trees(1, t, 19)
    c = R.Cache([n], 16, dtype, 20)
    for node in (3, 17, 39):
        slot = n - t + node
        c.v[c.table[0, slot // 16], slot % 16, 100] = math.inf
    q, q64 = queries(1, 3, t, dtype, 21)
    p = b.cache_params(1, 3, c.pages, 16, c.cols, tokens=t, dtype=dtype, flags=flags)
    out, lse = run(c, p, q, parents=par)
    check(c, p, q64, out, lse, [t], par)


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_large_logits(grkv_lib, dtype, flags):
    """The reference has to move many times, and far: keys that grow along the cache."""
    n = 1500
    c = R.Cache([n], 64, dtype, 22)
    grow = np.linspace(0.1, 40, n)
    for j in range(n):
        r = c.table[0, j // 64], j % 64
        c.k[r] = c.rounded(c.k[r] * grow[j])
    q, q64 = queries(1, 4, 9, dtype, 23)
    p = b.cache_params(1, 4, c.pages, 64, c.cols, tokens=9, dtype=dtype, flags=flags)
    out, lse = run(c, p, q)
    check(c, p, q64, out, lse, [9])


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_runs_are_equal_and_graphs_replay(grkv_lib, dtype, flags):
    c = R.Cache([3000, 100, 777], 32, dtype, 24)
    q, q64 = queries(3, 4, 20, dtype, 25)
    p = b.cache_params(3, 4, c.pages, 32, c.cols, tokens=20, dtype=dtype, flags=flags)
    o1, l1 = run(c, p, q)
    kd, vd = c.dev()
    dq, out = q.cuda(), torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.zeros(q.shape[:3], dtype=torch.float32, device="cuda")
    table, lens = R.int_dev(c.table), R.int_dev(c.lens)
    ws = [workspace(p), workspace(p)]
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [(out, lse), (torch.zeros_like(out), torch.zeros_like(lse))]
    for w, (o, l) in zip(ws, outs):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            b.grkv_attend(p, dq, kd, vd, table, lens, o, w, lse=l)
        graphs.append(gr)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):                  # both at once, each with its own workspace
        for o, l in outs:
            o.zero_()
            l.zero_()
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        torch.cuda.synchronize()
        for w, (o, l) in zip(ws, outs):
            assert torch.equal(o, o1) and torch.equal(l, l1)
            assert b.grkv_status(w) == b.GRKV_OK


def test_lse_is_optional_and_streams_are_honoured(grkv_lib):
    c = R.Cache([500], 16, "bf16", 26)
    q, q64 = queries(1, 4, 2, "bf16", 27)
    p = b.cache_params(1, 4, c.pages, 16, c.cols, tokens=2)
    st = torch.cuda.Stream()
    o1, _ = run(c, p, q, stream=st)
    kd, vd = c.dev()
    out, ws = torch.empty_like(o1), workspace(p)
    b.grkv_attend(p, q.cuda(), kd, vd, R.int_dev(c.table), R.int_dev(c.lens), out, ws)
    assert b.grkv_status(ws) == b.GRKV_OK and torch.equal(out, o1)


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_faulty_tables_lengths_and_parents_are_reported(grkv_lib, dtype, flags):
    """Nothing is read or written out of range; other units' results stand."""
    page = 16
    c = R.Cache([200, 150, 90], page, dtype, 28)
    q, q64 = queries(3, 2, 4, dtype, 29)
    p = b.cache_params(3, 2, c.pages, page, c.cols, tokens=4, dtype=dtype, flags=flags)
    kd, vd = c.dev()
    par = R.int_dev([[-1, 0, 1, 2]] * 3)
    good, _ = run(c, p, q, parents=[[-1, 0, 1, 2]] * 3)

    def status(table=None, lens=None, q_lens=None, parent=None):
        ws, out = workspace(p), torch.zeros(q.shape, dtype=q.dtype, device="cuda")
        b.grkv_attend_tree(p, q.cuda(), kd, vd, R.int_dev(c.table if table is None else table),
                           R.int_dev(lens or c.lens), par if parent is None else parent, out, ws,
                           q_lens=None if q_lens is None else R.int_dev(q_lens))
        st = b.grkv_status(ws)
        assert torch.equal(out[0], good[0])
        return st

    assert status() == b.GRKV_OK
    for entry in (-1, c.pages, 2 ** 31 - 1, -2 ** 31):
        t2 = c.table.copy()
        t2[1, 3] = entry
        assert status(table=t2) == b.GRKV_ERR_INVALID_ARG
    assert status(lens=[200, -5, 90]) == b.GRKV_ERR_INVALID_ARG
    assert status(lens=[200, 2 ** 31 - 1, 90]) == b.GRKV_ERR_INVALID_ARG
    assert status(q_lens=[4, 5, 4]) == b.GRKV_ERR_INVALID_ARG
    assert status(q_lens=[4, -1, 4]) == b.GRKV_ERR_INVALID_ARG
    for bad in (1, 3, 2 ** 31 - 1, -2):
        pr = R.int_dev([[-1, 0, 1, 2], [-1, bad, 1, 2], [-1, 0, 1, 2]])
        assert status(parent=pr) == b.GRKV_ERR_INVALID_ARG


@pytest.mark.parametrize("units,g,t,n,window", [(3, 4, 1500, 5000, 0), (2, 3, 3001, 3001, 500),
                                                (5, 1, 2100, 4500, 1000), (40, 8, 33, 2900, 700),
                                                (1, 8, 1024, 20000, 0)])
def test_long_chunks_agree_between_the_kernels(grkv_lib, units, g, t, n, window):
    """Runs of many slot tiles and many items to a CTA, where rings and parities wrap many
    times: tensor cores against CUDA cores, each within the bounds of its own arithmetic."""
    page = 32
    cols = R.pages_of(n, page)
    gen = torch.Generator(device="cuda").manual_seed(n)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float32, device="cuda", generator=gen).bfloat16()
    k, v, q = rnd(units * cols, page, D), rnd(units * cols, page, D), rnd(units, g, t, D)
    table = torch.randperm(units * cols, device="cuda", generator=gen).int().view(units, cols)
    lens = torch.tensor([n - 7 * u for u in range(units)], dtype=torch.int32, device="cuda")
    res = []
    for flags in (0, b.GRKV_FORCE_SIMT):
        p = b.cache_params(units, g, units * cols, page, cols, tokens=t, window=window, flags=flags)
        ws, out = workspace(p), torch.zeros_like(q)
        lse = torch.zeros(units, g, t, dtype=torch.float32, device="cuda")
        for _ in range(2):
            b.grkv_attend(p, q, k, v, table, lens, out, ws, lse=lse)
            assert b.grkv_status(ws) == b.GRKV_OK
        res.append((out.float(), lse))
    (o1, l1), (o2, l2) = res
    # A = sum_j p_j |v_j| is a mean of |v|, at most max |v| < 6 (few slots seen): both kernels
    # round the output (2^-8 |o| each), one rounds P (2^-8 A); the fp32 terms are below 2^-10 A
    mass = v.abs().max().item()
    assert ((o1 - o2).abs() <= 2.0 ** -7 * o2.abs() + (2.0 ** -8 + 2.0 ** -10) * mass).all()
    assert torch.equal(l1 == -math.inf, l2 == -math.inf)      # rows in front of a shorter cache
    assert (torch.where(l1 == l2, 0.0, l1 - l2).abs() <= 2.0 ** -9).all()


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_tables_of_many_columns(grkv_lib, dtype, flags):
    """A table that could hold more tiles than 32 bits count gives what a short one does."""
    g, t, page, n = 64, 2200, 128, 2300
    c = R.Cache([n], page, dtype, 40)
    q, _ = queries(1, g, t, dtype, 41)
    res = []
    for cols in (c.cols, 1 << 21):
        p = b.cache_params(1, g, c.pages, page, cols, tokens=t, dtype=dtype, flags=flags)
        table = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
        table[:, :c.cols] = R.int_dev(c.table)
        kd, vd = c.dev()
        out, ws = torch.zeros(q.shape, dtype=q.dtype, device="cuda"), workspace(p)
        lse = torch.zeros(q.shape[:3], dtype=torch.float32, device="cuda")
        b.grkv_attend(p, q.cuda(), kd, vd, table, R.int_dev(c.lens), out, ws, lse=lse)
        assert b.grkv_status(ws) == b.GRKV_OK
        res.append((out, lse))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def test_no_units(grkv_lib):
    p = b.cache_params(0, 1, 4, 16, 1)
    ws = workspace(p)
    z = torch.empty(0, dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros(4, 16, D, dtype=torch.bfloat16, device="cuda")
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    b.grkv_attend(p, z, pool, pool, e, e, z, ws)
    assert b.grkv_status(ws) == b.GRKV_OK
