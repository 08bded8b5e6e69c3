"""Rotated appends and turned compacts of long calls, far pages and many rows, bit for bit what the rows' operator
and the plain page operators give (whose values other tests hold to the formulas), and their status."""
import pytest
import torch

from paper_2605_31105_gb300 import binding as b

pytestmark = pytest.mark.gpu
D = 128
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rnd(gen, dtype, *shape):
    return torch.randn(*shape, dtype=torch.float32, device="cuda", generator=gen).to(TORCH[dtype])


class Cache:
    """Units of n slots in random pages of a pool whose content is random."""

    def __init__(self, dtype, u, n, page, seed, cols=None, g=4, tokens=1, spare=0):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        need = -(-n // page)
        cols = cols or need
        self.pages = u * need + spare
        self.order = torch.randperm(self.pages, device="cuda", generator=self.gen).int()
        self.table = torch.full((u, cols), -1, dtype=torch.int32, device="cuda")
        self.table[:, :need] = self.order[:u * need].view(u, need)
        self.lens = torch.full((u,), n, dtype=torch.int32, device="cuda")
        self.k, self.v = (rnd(self.gen, dtype, self.pages, page, D) for _ in range(2))
        self.p = b.cache_params(u, g, self.pages, page, cols, tokens=tokens, dtype=dtype)
        self.ws = torch.full((b.grkv_cache_workspace_size(self.p),), 0xFF, dtype=torch.uint8, device="cuda")


def same(x, y):
    word = torch.int16 if x.element_size() == 2 else torch.int32
    assert torch.equal(x.view(word), y.view(word))


# 50 MB and more: the status is cleared beside the kernel; below, by a memset; a few rows: by its cluster
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rotary,layout", [(128, "half"), (64, "pairs"), (20, "half")])
@pytest.mark.parametrize("u,t,g", [(8, 3000, 4), (40, 130, 5), (300, 3, 33), (3, 2, 1)])
def test_append(grkv_lib, dtype, rotary, layout, u, t, g):
    rope = b.grkv_rope_make(b.rope_params(rotary=rotary, layout=layout, scaling="yarn", factor=4.0))
    a, c = (Cache(dtype, u, t + 77, 32, u + t, g=g, tokens=t) for _ in range(2))
    k_new, v_new, q = (rnd(a.gen, dtype, *s) for s in ((u, t, D), (u, t, D), (u, g, t, D)))
    q_out, want, keys = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k_new)
    offset = torch.arange(u, dtype=torch.int32, device="cuda") * 1000
    b.grkv_cache_append_rope(a.p, rope, k_new, v_new, a.k, a.v, a.table, a.lens, a.ws, q=q, q_out=q_out, offset=offset)
    assert b.grkv_status(a.ws) == b.GRKV_OK
    b.grkv_rope_rows(rope, k_new[:, None], keys[:, None], start=offset + 77)
    b.grkv_rope_rows(rope, q, want, start=offset + 77)
    b.grkv_cache_append(c.p, keys, v_new, c.k, c.v, c.table, c.lens, c.ws)
    same(a.k, c.k)
    same(a.v, c.v)
    same(q_out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rotary,layout", [(128, "half"), (48, "pairs"), (20, "half")])
@pytest.mark.parametrize("u,n,t", [(200, 700, 600), (24, 1500, 1301), (6, 9000, 4200), (1000, 40, 33)])
@pytest.mark.parametrize("place", ["other", "in place"])
def test_compact(grkv_lib, dtype, rotary, layout, u, n, t, place):
    """Chunks of every size, blocks of one to many chunks and of 16 to 128 rows."""
    rope = b.grkv_rope_make(b.rope_params(rotary=rotary, layout=layout))
    other = place == "other"
    a, c = (Cache(dtype, u, n, 16, u + n, tokens=t, spare=u * -(-t // 16) if other else 0) for _ in range(2))
    kept = torch.rand(u, n, dtype=torch.float32, device="cuda", generator=a.gen).topk(t, 1).indices.sort(1).values
    idx, to = kept.int(), a.table
    if other:
        to = torch.full_like(a.table, -1)
        to[:, :-(-t // 16)] = a.order[u * -(-n // 16):].view(u, -1)
    before = [a.table.long().gather(1, kept // 16) * 16 + kept % 16]
    keys = a.k.view(-1, D)[before[0]]
    b.grkv_cache_compact_rope(a.p, rope, idx, a.k, a.v, a.table, a.lens, to, a.ws)
    assert b.grkv_status(a.ws) == b.GRKV_OK
    b.grkv_cache_compact(c.p, idx, c.k, c.v, c.table, c.lens, c.table if not other else to, c.ws)
    same(a.v, c.v)
    # the keys turned back by how far they have moved: the transposed rotation
    back = (kept - torch.arange(t, device="cuda")).int()
    b.grkv_rope_rows(rope, keys[:, None], keys[:, None], pos=back.contiguous(), transpose=True)
    dst = torch.arange(t, device="cuda")[None].expand(u, t)
    at = to.long().gather(1, dst // 16) * 16 + dst % 16
    c.k.view(-1, D)[at] = keys
    same(a.k, c.k)


@pytest.mark.parametrize("call", ["append", "compact", "shift", "map"])
@pytest.mark.parametrize("size", ["short", "long"])
def test_status_of_replayed_calls(grkv_lib, call, size):
    """A fault that comes and goes between replays of one captured call."""
    u, t = {"append": (16, 900), "compact": (16, 1100), "shift": (16, 1100), "map": (3000, 500)}[call]
    if size == "short":
        u, t = 16, 20
    cache = Cache("bf16", u, t + 16, 16, 1, tokens=t, spare=u * -(-t // 16), cols=-(-(t + 16) // 16))
    to = cache.table.clone()
    to[:, :-(-t // 16)] = cache.order[u * -(-(t + 16) // 16):].view(u, -1)
    rope = b.grkv_rope_make(b.rope_params())
    rows = rnd(cache.gen, "bf16", u, t, D) if call == "append" else None
    q = rnd(cache.gen, "bf16", u, 4, t, D) if call == "append" else None
    idx = (torch.arange(t, device="cuda")[None].expand(u, t) + 16).int().contiguous()
    pos, slot = torch.empty(u, t, dtype=torch.int32, device="cuda"), torch.empty(u, t, dtype=torch.int64, device="cuda")
    c = cache

    def go():
        if call == "append":
            b.grkv_cache_append_rope(c.p, rope, rows, rows, c.k, c.v, c.table, c.lens, c.ws, q=q, q_out=q)
        if call == "compact":
            b.grkv_cache_compact_rope(c.p, rope, idx, c.k, c.v, c.table, c.lens, to, c.ws)
        if call == "shift":
            b.grkv_cache_compact_rope(c.p, rope, idx, c.k, c.v, c.table, c.lens, c.table, c.ws)
        if call == "map":
            b.grkv_cache_map(c.p, c.table, c.lens, pos, slot, c.ws)

    go()
    assert b.grkv_status(c.ws) == b.GRKV_OK
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        go()
    entry = c.table[u - 1, 1].clone()
    for bad in (False, True, False, True, True, False):
        c.table[u - 1, 1] = -1 if bad else entry
        graph.replay()
        assert b.grkv_status(c.ws) == (b.GRKV_ERR_INVALID_ARG if bad else b.GRKV_OK)


def test_pages_beyond_32_bit_offsets(grkv_lib):
    """A pool of 2.3e9 elements of keys: rows appended to, kept in and attended over its last pages."""
    pages, page, n = 140000, 128, 300
    k, v = (torch.empty(pages, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(2)
    far, near = ints([[pages - 1, pages - 3, pages - 5]]), ints([[2, 0, 1]])
    rope = b.grkv_rope_make(b.rope_params())
    lens = ints([n])
    rows = [rnd(gen, "bf16", 1, n, D) for _ in range(2)]
    outs = []
    for table, out in ((far, ints([[pages - 7, pages - 9, pages - 11]])), (near, ints([[5, 4, 3]]))):
        p = b.cache_params(1, 1, pages, page, 3, tokens=n)
        ws = torch.empty(b.grkv_cache_workspace_size(p), dtype=torch.uint8, device="cuda")
        b.grkv_cache_append_rope(p, rope, *rows, k, v, table, lens, ws)
        assert b.grkv_status(ws) == b.GRKV_OK
        idx = torch.arange(20, 270, dtype=torch.int32, device="cuda")[None]
        p2 = b.cache_params(1, 1, pages, page, 3, tokens=250)
        b.grkv_cache_compact_rope(p2, rope, idx, k, v, table, lens, out, ws)
        pos, slot = torch.empty(1, 250, dtype=torch.int32, device="cuda"), torch.empty(1, 250, dtype=torch.int64, device="cuda")
        b.grkv_cache_map(p2, out, ints([250]), pos, slot, ws)
        assert b.grkv_status(ws) == b.GRKV_OK
        assert slot[0, 0].item() == out[0, 0].item() * page
        got = [x.view(-1, D)[slot[0]].clone() for x in (k, v)]
        for g, t in ((1, 1), (2, 1), (5, 1), (4, 3), (4, 40)):
            q = rnd(torch.Generator(device="cuda").manual_seed(g), "bf16", 1, g, t, D)
            p3 = b.cache_params(1, g, pages, page, 3, tokens=t)
            w3 = torch.empty(b.grkv_cache_workspace_size(p3), dtype=torch.uint8, device="cuda")
            o = torch.zeros_like(q)
            b.grkv_attend_cross(p3, q, k, v, out, ints([250]), o, w3)      # without lse
            assert b.grkv_status(w3) == b.GRKV_OK
            got.append(o)
        outs.append(got)
    for x, y in zip(*outs):
        same(x, y)
        assert x.float().abs().max() > 0
