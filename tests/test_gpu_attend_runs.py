"""grkv_attend and grkv_attend_tree where every CTA has a run of many slot tiles and several units: rings,
parities, moving references, masked tiles in the middle of runs, parts with references far
apart.  The plain form is torch in 64 bits; the bound is that of tests/cache_ref.py, with the term for P's
rounding to bf16 only where P is rounded: not in the CUDA-core kernels, and by 2^-16 where both
parts of it are multiplied."""
import math

import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
D = R.D
TYPES = [("f32", 0), ("bf16", 0), ("bf16", b.GRKV_FORCE_SIMT)]
# heads, tokens: items of 3, 8, 16, 50 and 60 rows, of 100 and 126 (one tile), of 300 (two tiles)
ROWS = [(3, 1), (8, 1), (4, 4), (50, 1), (5, 12), (50, 2), (3, 42), (60, 5)]


class Paged:
    """Units of the given lengths in random pages of a pool that is NaN elsewhere."""

    def __init__(self, lens, page, dtype, seed, shape=None):
        self.lens, self.page, self.dtype = [int(x) for x in lens], page, dtype
        gen = torch.Generator(device="cuda").manual_seed(seed)
        need = [R.pages_of(n, page) for n in self.lens]
        self.cols, self.pages = max(need) + 1, sum(need) + 3
        order = torch.randperm(self.pages, device="cuda", generator=gen).int()
        self.table = torch.full((len(lens), self.cols), -1, dtype=torch.int32, device="cuda")
        self.k, self.v = (torch.full((self.pages, page, D), math.nan, dtype=R.TORCH[dtype], device="cuda")
                          for _ in range(2))
        self.rows = []
        at = 0
        for u, n in enumerate(self.lens):
            self.table[u, :need[u]] = order[at:at + need[u]]
            rows = (order[at:at + need[u]].long()[:, None] * page
                    + torch.arange(page, device="cuda")).flatten()[:n]
            at += need[u]
            self.rows.append(rows)
            for pool, key in ((self.k, True), (self.v, False)):
                x = torch.randn(n, D, dtype=torch.float32, device="cuda", generator=gen)
                if key and shape is not None:
                    x *= shape(u, n)[:, None]
                pool.view(-1, D)[rows] = x.to(pool.dtype)
        self.dlens = R.int_dev(self.lens)

    def slots(self, u):
        return self.k.view(-1, D)[self.rows[u]].double(), self.v.view(-1, D)[self.rows[u]].double()

    def tiles(self):
        return sum(R.pages_of(n, 128) for n in self.lens)


def sees(n, t, window, sink, parent=None):
    """[t][n]: what token i of the last t of n slots sees."""
    j, i = torch.arange(n, device="cuda")[None], torch.arange(t, device="cuda")[:, None]
    base = n - t
    near = lambda at, pos: (at > pos - window) | (at < sink) if window else at == at
    if parent is None:
        return (j <= base + i) & near(j, base + i)
    dep = torch.tensor(R.depths(parent), device="cuda")
    see = ((j < base) & near(j, base + dep[:, None])).expand(t, n).clone()
    anc = torch.zeros(t, t, dtype=torch.bool)
    for a in range(t):
        if parent[a] >= 0:
            anc[a] = anc[parent[a]]
        anc[a, a] = True
    see[:, base:] = anc.cuda() & near(base + dep[None], base + dep[:, None])
    return see


def plain(q, k, v, see):
    """q [g][t][d] -> out, lse, mass, E by row; non-finite where a seen value or key is."""
    s = 1 / math.sqrt(D)
    x = (q @ k.T * s).masked_fill(~see, -math.inf)
    some = see.any(-1)
    w = torch.where(some[:, None], torch.softmax(x, -1), 0.0)
    fin = torch.where(v.isfinite(), v, 0.0)
    out, mass = w @ fin, w @ fin.abs()
    out += torch.where((see.double() @ (~v.isfinite()).double()) > 0, math.nan, 0.0)
    gam = (D + 2) * R.U32 / (1 - (D + 2) * R.U32)
    a = (q.abs() @ k.abs().nan_to_num(0).T * s).masked_fill(~see, 0.0).amax(-1)
    return out, torch.where(some, torch.logsumexp(x, -1), -math.inf), mass, gam * a


def run_and_check(c, g, t, flags, seed, window=0, sink=4, q_lens=None, parents=None, p_round=None):
    units, dtype = len(c.lens), c.dtype
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(units, g, t, D, dtype=torch.float32, device="cuda", generator=gen) * 1.5
    q = q.to(R.TORCH[dtype])
    p = b.cache_params(units, g, c.pages, c.page, c.cols, tokens=t, window=window, n_sink=sink,
                       dtype=dtype, flags=flags)
    ws = torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7), torch.full((units, g, t), 7, dtype=torch.float32, device="cuda")
    ql = None if q_lens is None else R.int_dev(q_lens)
    if parents is None:
        b.grkv_attend(p, q, c.k, c.v, c.table, c.dlens, out, ws, q_lens=ql, lse=lse)
    else:
        b.grkv_attend_tree(p, q, c.k, c.v, c.table, c.dlens, R.int_dev(parents), out, ws, q_lens=ql, lse=lse)
    assert b.grkv_status(ws) == b.GRKV_OK
    if p_round is None:
        p_round = 2.0 ** -8 if dtype == "bf16" and not flags else 0.0
    for u, n in enumerate(c.lens):
        m = t if q_lens is None else q_lens[u]
        assert (out[u, :, m:] == 7).all() and (lse[u, :, m:] == 7).all()
        if m == 0:
            continue
        got, got_lse = out[u, :, :m].double(), lse[u, :, :m].double()
        first = max(0, m - n)                        # rows in front of the cache see nothing
        assert (got[:, :first] == 0).all() and (got_lse[:, :first] == -math.inf).all()
        if first == m:
            continue
        k, v = c.slots(u)
        see = sees(n, m - first, window, sink, parents and parents[u][:m])
        o, z, mass, err = plain(q[u, :, first:m].double(), k, v, see)
        got, got_lse = got[:, first:], got_lse[:, first:]
        rel = 2 * err + (n + 64) * R.U32 + 2.0 ** -21
        tol = (rel + p_round)[..., None] * mass + R.ROUND[dtype] * o.abs()
        fine = o.isfinite()
        assert torch.equal(got.isfinite(), fine), f"unit {u}: non-finite elements"
        off = torch.where(fine, (got - o).abs() / tol.clamp_min(1e-300), 0.0)
        assert off.max() <= 1, f"unit {u} of {n} slots: {off.max():.2f} of the bound"
        ok = z.isfinite()
        assert torch.equal(got_lse.isfinite(), ok)
        assert ((got_lse - z).abs() <= rel + 4 * R.U32 * z.abs())[ok].all()


def long_runs(c):
    """More than three tiles to every CTA of a kernel that has two on each SM."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert c.tiles() > 3 * 2 * sms
    return c


def ragged(seed, units=96, lo=2500, hi=5000):
    """Long units with single tiles, single slots and empty units between them."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(lo, hi, units)
    lens[::5] = rng.integers(1, 129, len(lens[::5]))
    lens[::7] = 0
    lens[3::11] = 1
    return lens


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("window,sink", [(0, 4), (901, 70), (2000, 300)])
def test_ragged_units(grkv_lib, dtype, flags, g, t, window, sink):
    c = long_runs(Paged(ragged(t), 32, dtype, 1))
    rng = np.random.default_rng(2)
    q_lens = None if t == 1 else [int(x) for x in rng.integers(0, t + 1, len(c.lens))]
    run_and_check(c, g, t, flags, 3, window, sink, q_lens)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(3, 4), (4, 13), (5, 20), (4, 64)])
@pytest.mark.parametrize("window", [0, 1000])
def test_trees_over_ragged_units(grkv_lib, dtype, flags, g, t, window):
    rng = np.random.default_rng(4)
    c = long_runs(Paged(np.maximum(ragged(5), t), 16, dtype, 6))
    parents = [[max(-1, i - int(rng.integers(1, 6))) for i in range(t)] for _ in c.lens]
    run_and_check(c, g, t, flags, 7, window, 4, None, parents)


# Keys whose size changes along a unit: logits of 60 and more log2 units above and below the
# first tile's, of the largest keys up to some 350
SHAPES = {
    "growing": lambda u, n: torch.linspace(0.1, 40, n, device="cuda"),
    "falling": lambda u, n: torch.linspace(40, 0.1, n, device="cuda"),
    "waves": lambda u, n: 20 + 19 * torch.sin(torch.arange(n, device="cuda") * (0.004 + 0.001 * (u % 5))),
    "steps": lambda u, n: torch.where((torch.arange(n, device="cuda") // 300 + u) % 3 == 0, 40.0, 0.2),
}


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_references_that_move(grkv_lib, dtype, flags, g, t, shape):
    """Segments of eight tiles and more, of many units."""
    lens = [1500 - 7 * (u % 30) for u in range(112)]
    run_and_check(long_runs(Paged(lens, 64, dtype, 8, SHAPES[shape])), g, t, flags, 9)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(3, 1), (16, 1), (50, 1), (50, 2), (60, 5)])
@pytest.mark.parametrize("shape", ["growing", "falling", "waves"])
def test_parts_with_references_far_apart(grkv_lib, dtype, flags, g, t, shape):
    """Units that many CTAs hold parts of."""
    run_and_check(long_runs(Paged([50011, 41003, 45678], 128, dtype, 10, SHAPES[shape])), g, t, flags, 11)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("window,sink", [(0, 4), (400, 70)])
def test_values_and_keys_that_are_not_finite(grkv_lib, dtype, flags, g, t, window, sink):
    """In every unit a NaN or an infinity among the values, near its end, where its windows start, among
    the sinks or anywhere, and in some a NaN key; rows that see one are not finite."""
    c = long_runs(Paged([1500 - 7 * (u % 30) for u in range(112)], 32, dtype, 12))
    rng = np.random.default_rng(13)
    for u, n in enumerate(c.lens):
        spots = [n - 1 - int(rng.integers(0, t)),
                 min(n - 1, max(0, n - t - window + int(rng.integers(-40, 40)))),
                 int(rng.integers(0, 140)), int(rng.integers(0, n))]
        slot, col = spots[u % 4], int(rng.integers(0, D))
        c.v.view(-1, D)[c.rows[u][slot], col] = [math.nan, math.inf, -math.inf][u % 3]
        if u % 4 == 0:
            c.v.view(-1, D)[c.rows[u][spots[1]], (col + 3) % D] = -math.inf
        if u % 8 == 7:
            c.k.view(-1, D)[c.rows[u][spots[(u // 8) % 4]], col] = math.nan
    run_and_check(c, g, t, flags, 14, window, sink)


@pytest.mark.parametrize("g,t", [(1, 1), (8, 1), (16, 1), (64, 1), (4, 13), (2, 31)])
def test_both_parts_of_probabilities(grkv_lib, g, t):
    """bf16 on the tensor cores, up to 64 rows an item, one slot tile: P's rounding and what it leaves are
    both multiplied, 2^-16 of P remains."""
    c = Paged([1, 2, 15, 31, 64, 100, 127, 128] * 5, 16, "bf16", 15)
    run_and_check(c, g, t, 0, 16, p_round=2.0 ** -16)
