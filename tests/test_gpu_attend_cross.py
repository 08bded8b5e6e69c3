"""grkv_attend_cross against its formula in 64 bits, and a decoder's steps that use positions, slots, rotated
appends, both attentions and turned compactions together."""
import math

import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as R
from tests import rope_ref
from tests.test_gpu_attend import TYPES, queries, workspace

pytestmark = pytest.mark.gpu
D = R.D


def cross_unit(q, k, v, scale):
    """q [g][t][d], k, v [n][d] float64 -> out, lse, tolerance terms of cache_ref's docstring."""
    n = len(k)
    if n == 0:
        return np.zeros(q.shape), np.full(q.shape[:2], -math.inf), np.zeros(q.shape), np.zeros(q.shape[:2])
    x = q @ k.T * scale
    top = x.max(-1, keepdims=True)
    w = np.exp(x - top)
    p = w / w.sum(-1, keepdims=True)
    gam = (D + 2) * R.U32 / (1 - (D + 2) * R.U32)
    err = scale * gam * (np.abs(q) @ np.abs(k).T).max(-1)
    return p @ v, (top + np.log(w.sum(-1, keepdims=True)))[..., 0], p @ np.abs(v), err


def run(c, p, q, lens=None, q_lens=None, table=None):
    kd, vd = c.dev()
    out = torch.full(q.shape, 7, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:3], 7, dtype=torch.float32, device="cuda")
    ws = workspace(p)
    b.grkv_attend_cross(p, q.cuda(), kd, vd, R.int_dev(c.table if table is None else table),
                        R.int_dev(c.lens if lens is None else lens), out, ws,
                        q_lens=None if q_lens is None else R.int_dev(q_lens), lse=lse)
    return out, lse, b.grkv_status(ws)


def check(c, q64, out, lse, q_lens, scale=1 / math.sqrt(D)):
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for u, t in enumerate(q_lens):
        k, v = c.slots(u)
        o, z, mass, err = cross_unit(q64[u, :, :t], k, v, scale)
        rel = 2 * err + (len(k) + 64) * R.U32 + 2.0 ** -21
        tol = (rel + (2.0 ** -8 if c.dtype == "bf16" else 0))[..., None] * mass + R.ROUND[c.dtype] * np.abs(o)
        diff = np.abs(got[u, :, :t] - o)
        assert (diff <= tol).all(), (u, len(k), float((diff / np.maximum(tol, 1e-30)).max()))
        gl = got_lse[u, :, :t]
        if len(k) == 0:
            assert np.isneginf(gl).all()
        else:
            assert (np.abs(gl - z) <= rel + 4 * R.U32 * np.abs(z)).all()
        assert (got[u, :, t:] == 7).all() and (got_lse[u, :, t:] == 7).all(), "rows behind the last"


def case(lens, g, t, page, dtype, flags, q_lens=None, seed=0, **kw):
    c = R.Cache(lens, page, dtype, seed)
    q, q64 = queries(len(lens), g, t, dtype, seed + 1)
    p = b.cache_params(len(lens), g, c.pages, page, c.cols, tokens=t, dtype=dtype, flags=flags, **kw)
    out, lse, status = run(c, p, q, q_lens=q_lens)
    assert status == b.GRKV_OK
    check(c, q64, out, lse, q_lens or [t] * len(lens), kw.get("scale") or 1 / math.sqrt(D))


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_lengths(grkv_lib, dtype, flags, page):
    """Of 0, 1 and around pages and tiles; more queries than slots, and fewer."""
    lens = [1, 2, page - 1, page, page + 1, 127, 128, 129, 257, 1003, 0, 640]
    case(lens, 4, 1, page, dtype, flags)
    case(lens, 2, 37, page, dtype, flags, q_lens=[37, 0, 1, 2, 36, 37, 37, 37, 9, 37, 37, 5])


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(1, 1), (1, 300), (3, 5), (7, 41), (8, 33), (64, 1), (64, 5), (5, 130)])
def test_groups_and_tokens(grkv_lib, dtype, flags, g, t):
    case([300, 5, 0, 1, 1000, 131], g, t, 32, dtype, flags, seed=3)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(2, 1), (4, 70)])
def test_one_long_unit_is_split_over_the_ctas(grkv_lib, dtype, flags, g, t):
    case([30011], g, t, 64, dtype, flags, seed=4)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("seed", range(3))
def test_random_shapes(grkv_lib, dtype, flags, seed):
    rng = np.random.default_rng(50 + seed)
    for k in range(4):
        u, g = int(rng.integers(1, 9)), int(rng.integers(1, 17))
        t = int(rng.integers(1, 2400 // (u * g) + 2))
        case([int(x) for x in rng.integers(0, 900, u)], g, t, int(rng.choice([16, 32, 64, 128])), dtype, flags,
             q_lens=[int(x) for x in rng.integers(0, t + 1, u)], seed=100 * seed + k)


# rows 1 to 17 (a cluster a unit for up to 8 of fp32 and 16 of bf16, then tiles), clusters of 1 to 8 CTAs, status
# written by a unit's cluster (one unit), by a scan of all, and by units into a cleared word (600 units of 16
# columns)
@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(1, 1), (2, 1), (1, 2), (3, 1), (4, 1), (2, 2), (5, 1), (4, 2), (1, 7), (8, 1), (3, 3), (16, 1), (17, 1)])
@pytest.mark.parametrize("u,n", [(1, 1), (1, 255), (1, 900), (2, 1000), (40, 300), (130, 70), (600, 256)])
def test_few_rows(grkv_lib, dtype, flags, g, t, u, n):
    rng = np.random.default_rng(g * t + u)
    lens = [int(x) for x in rng.integers(0, n + 1, u)]
    lens[-1] = n
    q_lens = [int(x) for x in rng.integers(0, t + 1, u)]
    q_lens[-1] = t
    case(lens, g, t, 16, dtype, flags, q_lens=q_lens, seed=u)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("u", [1, 7, 600])
@pytest.mark.parametrize("fault", ["page", "below", "length", "negative", "rows"])
@pytest.mark.parametrize("g", [2, 5])
def test_faults_of_few_rows(grkv_lib, dtype, u, fault, g):
    """Reported, whichever unit has them; the units' other results stand."""
    rng = np.random.default_rng(u)
    lens = [int(x) for x in rng.integers(1, 200, u)]
    at = u // 2
    lens[at] = 208                               # the longest: whole pages, no more columns
    c = R.Cache(lens, 16, dtype, 40, spare=3)
    q, q64 = queries(u, g, 1, dtype, 41)
    p = b.cache_params(u, g, c.pages, 16, c.cols, dtype=dtype)
    table, given, q_lens, want = c.table.copy(), list(lens), [1] * u, [1] * u
    if fault in ("page", "below"):               # read as page 0
        table[at, 5] = c.pages if fault == "page" else -1
        c.k[0], c.v[0] = np.nan_to_num(c.k[0], nan=0.5), np.nan_to_num(c.v[0], nan=0.5)
        c.table[at, 5] = 0
    if fault == "length":
        given[at] = 209 + 1000
    if fault == "negative":
        given[at], c.lens[at] = -3, 0
    if fault == "rows":
        q_lens[at] = 2
    out, lse, status = run(c, p, q, lens=given, q_lens=q_lens, table=table)
    assert status == b.GRKV_ERR_INVALID_ARG
    check(c, q64, out, lse, want)
    out, lse, status = run(c, p, q, lens=[min(max(x, 0), 208) for x in given])   # and the next call is clean
    assert status == b.GRKV_OK
    check(c, q64, out, lse, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g", [2, 7])
def test_calls_of_few_rows_are_equal_and_replay_beside_others(grkv_lib, dtype, g):
    """Two captured calls of one workspace one after the other, and of two workspaces at once."""
    c = R.Cache([1500, 3, 0, 777, 1024], 32, dtype, 42)
    q, q64 = queries(5, g, 1, dtype, 43)
    p = b.cache_params(5, g, c.pages, 32, c.cols, dtype=dtype)
    o1, l1, _ = run(c, p, q)
    kd, vd = c.dev()
    dq, table, lens = q.cuda(), R.int_dev(c.table), R.int_dev(c.lens)
    ws = [workspace(p), workspace(p)]
    outs = [(torch.zeros_like(o1), torch.zeros_like(l1)) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for w, (o, l) in zip((ws[0], ws[0], ws[1]), outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            b.grkv_attend_cross(p, dq, kd, vd, table, lens, o, w, lse=l)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for o, l in outs:
            o.zero_()
            l.zero_()
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        with torch.cuda.stream(other):
            graphs[2].replay()
        torch.cuda.synchronize()
        for o, l in outs:
            assert torch.equal(o, o1) and torch.equal(l, l1)
        assert b.grkv_status(ws[0]) == b.grkv_status(ws[1]) == b.GRKV_OK


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_a_window_is_not_read(grkv_lib, dtype, flags):
    case([900, 3], 2, 9, 16, dtype, flags, seed=5, window=20, n_sink=2)


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_scale(grkv_lib, dtype, flags):
    case([200, 90], 2, 3, 16, dtype, flags, seed=8, scale=0.25)


@pytest.mark.parametrize("dtype,flags,g", [("bf16", 0, 20), ("bf16", b.GRKV_FORCE_SIMT, 20),
                                           ("f32", b.GRKV_FORCE_SIMT, 20), ("f32", 0, 7)])
def test_one_token_sees_what_decoding_sees(grkv_lib, dtype, flags, g):
    """The last slot's own token sees every slot: bit for bit grkv_attend, where its kernels run."""
    c = R.Cache([1, 77, 4000, 333], 32, dtype, 9)
    q, _ = queries(4, g, 1, dtype, 10)
    p = b.cache_params(4, g, c.pages, 32, c.cols, dtype=dtype, flags=flags)
    out, lse, _ = run(c, p, q)
    kd, vd = c.dev()
    o, l, ws = torch.zeros_like(out), torch.zeros_like(lse), workspace(p)
    b.grkv_attend(p, q.cuda(), kd, vd, R.int_dev(c.table), R.int_dev(c.lens), o, ws, lse=l)
    assert torch.equal(out, o) and torch.equal(lse, l)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(1, 1), (2, 1), (5, 1), (4, 3), (4, 100)])
def test_what_lies_behind_the_length_stays_out(grkv_lib, dtype, flags, g, t):
    """Values of NaN and infinities behind the last slot of a page, pages that are not there."""
    c = R.Cache([301, 0, 640], 128, dtype, 11, extra_cols=2)
    for what in (math.nan, math.inf, -math.inf):
        row = c.table[0, 2]
        c.k[row, 301 - 256:], c.v[row, 301 - 256:] = what, what
        q, q64 = queries(3, g, t, dtype, 12)
        p = b.cache_params(3, g, c.pages, 128, c.cols, tokens=t, dtype=dtype, flags=flags)
        out, lse, status = run(c, p, q)
        assert status == b.GRKV_OK and (c.table[:, -1] == -1).all()
        check(c, q64, out, lse, [t] * 3)


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(1, 1), (2, 1), (5, 1), (4, 3), (2, 70)])
def test_what_a_row_sees_reaches_it(grkv_lib, dtype, flags, g, t):
    """A value that is not finite, in a whole tile and in the last one, reaches every row's element."""
    for slot in (3, 299):
        for what in (math.nan, math.inf):
            c = R.Cache([300], 16, dtype, 13)
            c.v[c.table[0, slot // 16], slot % 16, 9] = what
            q, _ = queries(1, g, t, dtype, 14)
            p = b.cache_params(1, g, c.pages, 16, c.cols, tokens=t, dtype=dtype, flags=flags)
            out, _, _ = run(c, p, q)
            assert not torch.isfinite(out[..., 9]).any()
            assert torch.isfinite(out[..., :9]).all() and torch.isfinite(out[..., 10:]).all()
            c.v[c.table[0, slot // 16], slot % 16, 9] = 0.0
            c.k[c.table[0, slot // 16], slot % 16, 5] = math.nan     # a key of NaN: every element
            out, _, _ = run(c, p, q)
            assert torch.isnan(out).all()


@pytest.mark.parametrize("dtype,flags", TYPES)
@pytest.mark.parametrize("g,t", [(4, 90), (1, 1), (2, 1), (7, 1), (4, 4)])
def test_large_logits(grkv_lib, dtype, flags, g, t):
    """Keys that grow along the cache; then logits of up to 2^40, which leave every row its largest one's value."""
    c = R.Cache([1500], 64, dtype, 22)
    grow = np.linspace(0.1, 40, 1500)
    for j in range(1500):
        r = c.table[0, j // 64], j % 64
        c.k[r] = c.rounded(c.k[r] * grow[j])
    q, q64 = queries(1, g, t, dtype, 23)
    p = b.cache_params(1, g, c.pages, 64, c.cols, tokens=t, dtype=dtype, flags=flags)
    out, lse, _ = run(c, p, q)
    check(c, q64, out, lse, [t])
    p.scale = 2.0 ** 28
    out, lse, _ = run(c, p, q)
    k, v = c.slots(0)
    x = q64[0] @ k.T                                          # the two largest are far apart in most rows
    top = np.sort(x, -1)
    clear = top[..., -1] - top[..., -2] > 1e-3 * np.abs(x).max()
    best = v[x.argmax(-1)]
    got = out[0].double().cpu().numpy()
    assert clear.mean() > 0.5 and torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert np.abs(got - best)[clear].max() <= R.ROUND[dtype] * np.abs(best).max()


@pytest.mark.parametrize("dtype,flags", TYPES)
def test_faults_are_reported(grkv_lib, dtype, flags):
    """Lengths past the table count as its end, missing pages are read as page 0."""
    c = R.Cache([100, 64], 32, dtype, 15, spare=0)
    q, q64 = queries(2, 2, 3, dtype, 16)
    p = b.cache_params(2, 2, c.pages, 32, c.cols, tokens=3, dtype=dtype, flags=flags)
    out, lse, status = run(c, p, q, q_lens=[3, 4])
    assert status == b.GRKV_ERR_INVALID_ARG
    check(c, q64, out, lse, [3, 3])
    table = c.table.copy()
    table[1, 0] = c.pages
    c.table[1, 0] = 0
    for page in range(c.pages):          # page 0 may be a unit's last one, with slots that are not filled
        hole = np.isnan(c.k[page])
        c.k[page][hole] = c.v[page][hole] = 0.5
    out, lse, status = run(c, p, q, table=table)
    assert status == b.GRKV_ERR_INVALID_ARG
    check(c, q64, out, lse, [3, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,t", [(20, 1), (50, 2), (4, 200)])
def test_a_wait_that_runs_out_ends_the_call(grkv_lib, dtype, g, t):
    gen = torch.Generator(device="cuda").manual_seed(g)
    rnd = lambda *s: torch.randn(*s, dtype=torch.float32, device="cuda", generator=gen).to(R.TORCH[dtype])
    k, v, q = rnd(60, 64, D), rnd(60, 64, D), rnd(300, g, t, D)
    table = torch.arange(60, device="cuda").int().repeat(300, 1)
    lens = torch.full((300,), 60 * 64 - 5, dtype=torch.int32, device="cuda")
    p = b.cache_params(300, g, 60, 64, 60, tokens=t, dtype=dtype)
    ws, outs = workspace(p), []
    for flags in (0, b.GRKV_TEST_TIMEOUT, 0):
        p.flags = flags
        out = torch.zeros_like(q)
        b.grkv_attend_cross(p, q, k, v, table, lens, out, ws)
        assert b.grkv_status(ws) == (b.GRKV_ERR_TIMEOUT if flags else b.GRKV_OK)
        if not flags:
            outs.append(out)
    assert outs[0].abs().max() > 0 and torch.equal(*outs)


# fp32 rows of 9 and more are products of bf16 parts; of the other kernels, for comparison
@pytest.mark.parametrize("flags", [0, b.GRKV_FORCE_SIMT])
@pytest.mark.parametrize("g,t", [(9, 1), (4, 70), (33, 4), (64, 3), (1, 129)])
@pytest.mark.parametrize("power_k,power_v", [(0, 100), (0, -100), (40, 0), (-40, 60)])
def test_numbers_of_any_size(grkv_lib, flags, g, t, power_k, power_v):
    """Values near the ends of fp32's range, one at its very end; keys that the queries' size makes up for."""
    c = R.Cache([300, 77, 64, 0], 16, "f32", 50)
    q, q64 = queries(4, g, t, "f32", 51)
    q, q64 = q * 2.0 ** -power_k, q64 * 2.0 ** -power_k
    c.k, c.v = c.k * 2.0 ** power_k, c.v * 2.0 ** power_v
    if power_v > 0:
        c.v[c.table[1, 3], 9, 17] = float(np.finfo(np.float32).max)
    p = b.cache_params(4, g, c.pages, 16, c.cols, tokens=t, dtype="f32", flags=flags)
    out, lse, status = run(c, p, q)
    assert status == b.GRKV_OK
    check(c, q64, out, lse, [t] * 4)


@pytest.mark.parametrize("g,t", [(9, 1), (7, 77), (4, 200)])
def test_fp32_runs_are_equal(grkv_lib, g, t):
    """Many units, so that a CTA has several segments, whole ones and parts; twice the same to the bit."""
    rng = np.random.default_rng(60)
    lens = [int(x) for x in rng.integers(0, 700, 60)]
    c = R.Cache(lens, 32, "f32", 61)
    q, q64 = queries(60, g, t, "f32", 62)
    q_lens = [int(x) for x in rng.integers(0, t + 1, 60)]
    p = b.cache_params(60, g, c.pages, 32, c.cols, tokens=t, dtype="f32")
    o1, l1, status = run(c, p, q, q_lens=q_lens)
    assert status == b.GRKV_OK
    check(c, q64, o1, l1, q_lens)
    o2, l2, _ = run(c, p, q, q_lens=q_lens)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


# ---------------------------------------------------------------- a decoder's steps
def self_unit(q, k, v):
    """One token over every slot."""
    return cross_unit(q[:, None], k, v, 1 / math.sqrt(D))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("captured", [False, True])
def test_a_decoder_with_encoder_states(grkv_lib, dtype, captured):
    """Units that a compression shortened (positions ahead of slots) decode six tokens beside encoder
    states in the same pool; after the third, all but the first four and the last 40 slots are evicted in
    place, keys turned to their new slots.  The step is captured once and replayed, too."""
    page, g, u = 16, 2, 3
    lens, enc, ahead = [70, 61, 100], [33, 200, 1], np.array([5000, 0, 131072])
    c = R.Cache(lens + enc, page, dtype, 30, spare=30, extra_cols=4)
    layout, kw = "half", dict(rotary=64, scaling="yarn", factor=8.0, original=4096.0)
    rope = b.grkv_rope_make(b.rope_params(layout=layout, **kw))
    p = b.cache_params(u, g, c.pages, page, c.cols, dtype=dtype)
    pk = b.cache_params(u, g, c.pages, page, c.cols, tokens=44, dtype=dtype)
    ws = workspace(pk)                       # for the longest of the calls
    kd, vd = c.dev()
    table, e_table = R.int_dev(c.table[:u]), R.int_dev(c.table[u:])
    refs, e_lens = R.int_dev(c.refs), R.int_dev(enc)
    rt = R.TORCH[dtype]
    row = lambda *s: torch.zeros(*s, D, dtype=rt, device="cuda")
    held, now, offset = R.int_dev(lens), R.int_dev(lens), R.int_dev(ahead)
    pos = torch.zeros(u, 1, dtype=torch.int32, device="cuda")
    slot = torch.zeros(u, 1, dtype=torch.int64, device="cuda")
    k_new, v_new, q, q_rot, out, x_out = row(u, 1), row(u, 1), row(u, g, 1), row(u, g, 1), row(u, g, 1), row(u, g, 1)
    cross_p = b.cache_params(u, g, c.pages, page, c.cols, dtype=dtype)
    codes = []

    def step(check=True):
        now.add_(1)
        for call in (lambda: b.grkv_cache_reserve(p, table, held, now, refs, kd, vd, ws),
                     lambda: b.grkv_cache_map(p, table, now, pos, slot, ws, offset=offset),
                     lambda: b.grkv_cache_append_rope(p, rope, k_new, v_new, kd, vd, table, now, ws, q=q,
                                                      q_out=q_rot, pos=pos),
                     lambda: b.grkv_attend(p, q_rot, kd, vd, table, now, out, ws),
                     lambda: b.grkv_attend_cross(cross_p, q, kd, vd, e_table, e_lens, x_out, ws)):
            call()
            if check:
                codes.append(b.grkv_status(ws))
        held.copy_(now)

    # the reference: the units' keys and values as they lie in the cache
    ks, vs = zip(*[[x.copy() for x in c.slots(x)] for x in range(u)])
    ks, vs = list(ks), list(vs)
    es = [c.slots(u + x, enc[x]) for x in range(u)]
    rng = np.random.default_rng(31)
    replay = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        replay = torch.cuda.CUDAGraph()
        with torch.cuda.graph(replay, stream=side):
            step(check=False)
    # attention's bound, and what the rotated keys' own errors (half a step of the type on rows of norm
    # ~11 times queries of norm ~17, over sqrt(d)) add to logits: R |q| |k| / 11.3, twice in a probability
    half = R.ROUND[dtype]
    for n in range(6):
        fresh = [torch.from_numpy(rng.standard_normal(s)).to(rt) for s in ((u, 1, D), (u, 1, D), (u, g, 1, D))]
        for t, x in zip((k_new, v_new, q), fresh):
            t.copy_(x)
        if captured:
            replay.replay()
        else:
            step()
        want_pos = [len(ks[x]) + int(ahead[x]) for x in range(u)]
        assert pos.flatten().tolist() == want_pos
        fk, fv, fq = (x.double().numpy() for x in fresh)
        for x in range(u):
            new, _ = rope_ref.rotate(fk[x], [want_pos[x]], layout, **kw)
            ks[x], vs[x] = np.concatenate([ks[x], new]), np.concatenate([vs[x], fv[x]])
            rq, _ = rope_ref.rotate(fq[x, :, 0], np.full(g, want_pos[x]), layout, **kw)
            for got, (o, _, mass, err), qq, kk in (
                    (out, self_unit(rq, ks[x], vs[x]), rq, ks[x]),
                    (x_out, self_unit(fq[x, :, 0], *es[x]), fq[x, :, 0], es[x][0])):
                drift = 4 * half * (np.abs(qq) @ np.abs(kk).T).max() / math.sqrt(D)
                rel = 2 * err + (len(kk) + 64) * R.U32 + 2.0 ** -21 + (2.0 ** -8 if dtype == "bf16" else 0)
                tol = (rel[..., None] + 2 * drift) * mass + half * np.abs(o)
                diff = np.abs(got[x].double().cpu().numpy() - o)
                assert (diff <= tol).all(), (n, x, float((diff / tol).max()))
        if n == 2:
            idx = np.stack([np.concatenate([np.arange(4), np.arange(len(k) - 40, len(k))]) for k in ks])
            b.grkv_cache_compact_rope(pk, rope, R.int_dev(idx), kd, vd, table, now, table, ws)
            assert b.grkv_status(ws) == b.GRKV_OK
            now.fill_(44)
            held.fill_(44)
            b.grkv_cache_trim(p, table, now, refs, ws)
            for x in range(u):
                ks[x], _ = rope_ref.rotate(ks[x][idx[x]], np.arange(44) - idx[x], layout, amplitude=1.0, **kw)
                vs[x] = vs[x][idx[x]]
    assert not any(codes)
