"""Positions and slots of new rows against plain bookkeeping."""
import numpy as np
import pytest
import torch

from paper_2605_31105_gb300 import binding as b
from tests import cache_ref as C

pytestmark = pytest.mark.gpu


def run(table, lens, pages, page, t, count=None, parent=None, offset=None, packed=False, code=b.GRKV_OK):
    u, cols = table.shape
    p = b.cache_params(u, 1, pages, page, cols, tokens=t)
    ws = torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")
    pos = torch.full((u, t), 77, dtype=torch.int32, device="cuda")
    slot = torch.full((u, t), 77, dtype=torch.int64, device="cuda")
    first = torch.full((u + 1,), 77, dtype=torch.int64, device="cuda") if packed else None
    dev = lambda x: None if x is None else C.int_dev(x)
    b.grkv_cache_map(p, C.int_dev(table), C.int_dev(lens), pos, slot, ws, count=dev(count), parent=dev(parent),
                     offset=dev(offset), first_row=first)
    assert b.grkv_status(ws) == code
    return pos.cpu().numpy(), slot.cpu().numpy(), None if first is None else first.cpu().numpy()


def plain(table, lens, pages, page, t, count=None, parent=None, offset=None, packed=False):
    u, cols = table.shape
    count = [t] * u if count is None else [min(max(int(x), 0), t) for x in count]
    pos, slot = np.full((u, t), -1, np.int32), np.full((u, t), -1, np.int64)
    first = np.concatenate([[0], np.cumsum(count)])
    for x in range(u):
        for i in range(count[x]):
            s = int(lens[x]) - count[x] + i
            ahead = i
            if parent is not None:
                ahead, node = 0, parent[x][i]
                while node >= 0:
                    ahead, node = ahead + 1, parent[x][node]
            p = int(lens[x]) - count[x] + ahead + (0 if offset is None else int(offset[x]))
            row = -1
            if 0 <= s < cols * page and 0 <= table[x, s // page] < pages:
                row = int(table[x, s // page]) * page + s % page
            at = divmod(int(first[x]) + i, t) if packed else (x, i)
            pos[at], slot[at] = (p if 0 <= p < 1 << 31 else -1), row
    return pos, slot, first if packed else None


def same(*a, code=b.GRKV_OK, **kw):
    for got, want in zip(run(*a, code=code, **kw), plain(*a, **kw)):
        assert np.array_equal(got, want)


def pool(u, page, t, n, seed, spare=5):
    rng = np.random.default_rng(seed)
    lens = rng.integers(t, n + 1, u)
    cols = C.pages_of(int(lens.max()), page) + 1
    need = [C.pages_of(int(x), page) for x in lens]
    order = rng.permutation(sum(need) + spare)
    table = np.full((u, cols), -1, np.int32)
    at = 0
    for x in range(u):
        table[x, :need[x]] = order[at:at + need[x]]
        at += need[x]
    return table, lens, len(order), rng


# one block and several, units of one row, of a block's rows, of more, of odd numbers
@pytest.mark.parametrize("u,t", [(1, 1), (1, 1023), (3, 1024), (2, 1025), (2, 3000), (7, 13), (300, 5), (1023, 1),
                                 (1025, 1), (4096, 1), (4097, 1), (5000, 1), (2600, 3), (9000, 7)])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("page", [16, 128])
def test_map(grkv_lib, u, t, packed, page):
    table, lens, pages, rng = pool(u, page, t, t + 300, u + t)
    count = rng.integers(0, t + 1, u)
    count[rng.integers(u)] = 0
    offset = rng.integers(0, 1 << 20, u)
    same(table, lens, pages, page, t, packed=packed)
    same(table, lens, pages, page, t, count=count, offset=offset, packed=packed)
    same(table, lens, pages, page, t, count=np.zeros(u, int), packed=packed)


@pytest.mark.parametrize("u,t", [(1, 1), (3, 2), (40, 64), (9, 256), (33, 31), (5, 255), (200, 17)])
@pytest.mark.parametrize("packed", [False, True])
def test_trees(grkv_lib, u, t, packed):
    table, lens, pages, rng = pool(u, 16, t, t + 300, u * t)
    parent = np.array([[max(-1, i - int(rng.integers(1, 6))) for i in range(t)] for _ in range(u)])
    parent[0] = np.arange(t) - 1          # a chain: as deep as it gets
    if u > 1:
        parent[1] = -1
    count = rng.integers(0, t + 1, u)
    count[0] = t
    same(table, lens, pages, 16, t, parent=parent, offset=rng.integers(0, 99, u), packed=packed)
    parent[np.arange(t)[None] >= count[:, None]] = 12345        # of nodes that are not there
    same(table, lens, pages, 16, t, parent=parent, count=count, packed=packed)


@pytest.mark.parametrize("u", [6, 3000])
def test_faults_are_reported(grkv_lib, u):
    """In one block, which writes the status, and in several."""
    inv = b.GRKV_ERR_INVALID_ARG
    table, lens, pages, rng = pool(u, 16, 4, 60, 1)
    t = 4
    bad = table.copy()
    bad[2, (lens[2] - 1) // 16] = -1
    bad[u - 1, (lens[u - 1] - 1) // 16] = pages
    same(bad, lens, pages, 16, t, code=inv)
    long = lens.copy()
    long[1], long[3], long[4] = table.shape[1] * 16 + 2, 2, -5
    same(table, long, pages, 16, t, code=inv)
    count = np.full(u, 3)
    count[0], count[u - 1] = -1, 5
    same(table, lens, pages, 16, t, count=count, code=inv)
    same(table, lens, pages, 16, t, count=count, code=inv, packed=True)
    offset = np.zeros(u, np.int64)
    offset[0], offset[1] = -int(lens[0]) + 2, 2 ** 31 - 1
    same(table, lens, pages, 16, t, offset=offset, code=inv)
    parent = np.tile(np.arange(t) - 1, (u, 1))
    parent[2, 1], parent[3, 3] = 1, -2                # a node's own, below none: taken as none
    pos, slot, _ = run(table, lens, pages, 16, t, parent=parent, code=inv)
    parent[2, 1], parent[3, 3] = -1, -1
    want = plain(table, lens, pages, 16, t, parent=parent)
    assert np.array_equal(pos, want[0]) and np.array_equal(slot, want[1])


def test_no_units(grkv_lib):
    p = b.cache_params(0, 1, 4, 16, 1)
    ws = torch.full((b.grkv_cache_workspace_size(p),), 0xFF, dtype=torch.uint8, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    first = torch.full((1,), 77, dtype=torch.int64, device="cuda")
    b.grkv_cache_map(p, none, none, none, none.long(), ws, first_row=first)
    assert b.grkv_status(ws) == b.GRKV_OK and first.item() == 0
