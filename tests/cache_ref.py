"""Plain forms of the paged cache's operators in numpy and 64 bits, and seeded caches.

Tolerances of the attention follow from its arithmetic.  A logit is an fp32 sum of d exact
or once-rounded products times the scale: off by at most E = s gamma_(d+2) sum |q k|.  A
probability then has a relative error of 2 E, plus the exponential's and the reference's
roundings (2^-21), plus n u for the fp32 sums over n slots.  bf16 rounds each probability
(2^-8) and the output (2^-8); fp32 rounds the output (2^-24).  So with
A = sum_j p_j |v_j|:  |out - o| <= (2 E + (n + 64) u + 2^-21 [+ 2^-8]) A + round |o|.
"""
import math

import numpy as np
import torch

D = 128
U32 = 2.0 ** -24
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def pages_of(n, page):
    return -(-n // page)


def depths(parent):
    d = []
    for i, p in enumerate(parent):
        d.append(d[p] + 1 if p >= 0 else 0)
    return d


def visible(n, t, i, window, sink, parent=None):
    """Slots that token i of the last t of n slots sees."""
    base = n - t
    see = np.zeros(max(n, 0), bool)
    if parent is None:
        pos, slots = base + i, {j: j for j in range(0, base + i + 1)}
    else:
        dep = depths(parent)
        pos, slots = base + dep[i], {j: j for j in range(0, base)}
        x = i
        while x >= 0:
            slots[base + x] = base + dep[x]
            x = parent[x]
    for j, at in slots.items():
        if j >= 0 and (window == 0 or at > pos - window or at < sink):
            see[j] = True
    return see


def attend_unit(q, k, v, q_len, window, sink, scale=None, parent=None):
    """q [g][t][d], k, v [n][d] float64 -> out, lse, tolerance terms (A, E), by row."""
    g, t, _ = q.shape
    n = k.shape[0]
    s = 1.0 / math.sqrt(D) if scale is None else scale
    out, lse = np.zeros((g, t, D)), np.full((g, t), -math.inf)
    mass, err = np.zeros((g, t, D)), np.zeros((g, t))
    for i in range(q_len):
        see = visible(n, q_len, i, window, sink, parent)
        if not see.any():
            continue
        kk, vv = k[see], v[see]
        for h in range(g):
            with np.errstate(all="ignore"):
                x = kk @ q[h, i] * s
                top = x.max()
                if np.isneginf(top):
                    continue
                w = np.exp(x - top)
                p = w / w.sum()
                out[h, i] = p @ vv
                lse[h, i] = top + math.log(w.sum()) if np.isfinite(w.sum()) else math.nan
                mass[h, i] = p @ np.abs(vv)
                gam = (D + 2) * U32 / (1 - (D + 2) * U32)
                err[h, i] = s * gam * (np.abs(kk) @ np.abs(q[h, i])).max()
    return out, lse, mass, err


class Cache:
    """A pool whose unused slots are NaN, with units of the given lengths in random pages."""

    def __init__(self, lens, page, dtype, seed, spare=5, extra_cols=0):
        rng = np.random.default_rng(seed)
        self.page, self.dtype, self.lens = page, dtype, list(lens)
        self.cols = max(1, max((pages_of(n, page) for n in lens), default=1) + extra_cols)
        used = sum(pages_of(n, page) for n in lens)
        self.pages = used + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(lens), self.cols), -1, np.int32)
        self.k = np.full((self.pages, page, D), np.nan)
        self.v = np.full((self.pages, page, D), np.nan)
        at = 0
        for u, n in enumerate(lens):
            for c in range(pages_of(n, page)):
                self.table[u, c] = p = order[at]
                at += 1
                m = min(page, n - c * page)
                self.k[p, :m] = self.rounded(rng.standard_normal((m, D)))
                self.v[p, :m] = self.rounded(rng.standard_normal((m, D)))
        self.refs = np.bincount(self.table[self.table >= 0], minlength=self.pages).astype(np.int32)

    def rounded(self, x):
        return torch.from_numpy(np.asarray(x)).to(TORCH[self.dtype]).double().numpy()

    def slots(self, u, n=None, table=None):
        n = self.lens[u] if n is None else n
        table = self.table if table is None else table
        row = table[u, :pages_of(n, self.page)].clip(0)
        return (self.k[row].reshape(-1, D)[:n], self.v[row].reshape(-1, D)[:n])

    def dev(self):
        as_t = lambda x: torch.from_numpy(x).to(TORCH[self.dtype]).cuda()
        return as_t(self.k), as_t(self.v)


def int_dev(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


# ------------------------------------------------------------------ page operators
def reserve(table, lens, want, refs, k, v, page):
    """In place; False (and nothing changed) if the pool has too few free pages."""
    before = refs.copy()
    free = [p for p in range(len(refs)) if refs[p] <= 0]
    todo = []
    for u in range(len(lens)):
        if want[u] > lens[u]:
            for c in range(lens[u] // page, pages_of(want[u], page)):
                e = table[u, c]
                if e < 0 or before[e] > 1:
                    todo.append((u, c, int(e)))
    if len(todo) > len(free):
        return False
    for (u, c, old), new in zip(todo, free):
        if old >= 0:
            refs[old] -= 1
            part = lens[u] - c * page
            if part > 0:
                k[new, :part], v[new, :part] = k[old, :part], v[old, :part]
        refs[new] = 1
        table[u, c] = new
    return True


def fork(src, table_in, lens_in, refs, cols, page):
    table = np.full((len(src), cols), -1, np.int32)
    lens = np.zeros(len(src), np.int32)
    for u, s in enumerate(src):
        if s >= 0:
            lens[u] = lens_in[s]
            m = pages_of(lens[u], page)
            table[u, :m] = table_in[s, :m]
            np.add.at(refs, table[u, :m], 1)
    return table, lens


def trim(table, lens, refs, page):
    for u in range(len(lens)):
        for c in range(pages_of(lens[u], page), table.shape[1]):
            if table[u, c] >= 0:
                refs[table[u, c]] -= 1
                table[u, c] = -1


def at(table, u, slot, page):
    return table[u, slot // page], slot % page
