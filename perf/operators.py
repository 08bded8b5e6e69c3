"""The measured work of the paged cache: its page operators and the attention that reads it.

A case is one pass through one operator (or, for `beam` and `draft`, through the calls
that a decoding step makes of them).  `op` names it:

  attend   grkv_attend: queries of the last `tokens` slots of each unit over its pages, with
           a sliding window and sinks (window 0: every earlier slot).  tokens 1 is decoding,
           more is a chunk of prefill
  tree     grkv_attend_tree: `tokens` drafted nodes of each unit over its pages and each other
  compact  grkv_cache_compact: the kept slots of a retained set, moved to pages of their own
  append   grkv_cache_append: `tokens` new rows of each unit into its pages
  beam     a step of beam search: the last step's beams dropped (grkv_cache_trim), the chosen
           ones forked (grkv_cache_fork), pages for the new token (grkv_cache_reserve, with
           copies of shared pages), its rows appended
  draft    a step of speculative decoding: the last draft dropped, the cache forked, pages for
           `tokens` drafted rows, their append, tree attention, the accepted path moved
           together in place (grkv_cache_compact), the rest of the pages dropped

Sizes: units U = batch x KV heads (x layers), g query heads per KV head, head size 128, `n`
the longest unit, `page` slots per page.  `ragged` units hold between n / 16 and n slots
(always the same ones for a case), as budgets per unit and sequences of a batch do.  Pages
lie in the pool in random order.  The first slots are sinks: keys that every query favours.
"""
import math

import torch

own = False

D = 128
_DEFAULTS = dict(op="attend", dtype="bf16", units=8, group=4, tokens=1, n=8192, ragged=False,
                 page=64, window=0, sink=4, beams=1, keep=0)


def _case(**kw):
    return dict(_DEFAULTS, **kw)


def listed():
    return [
        # One KV head after a short prompt, one query: the smallest call, latency.
        _case(name="decode_head_1k", units=1, group=1, n=1003, page=16),
        # One layer of a batch of eight sequences with budgets per head: ordinary decoding.
        _case(name="decode_ragged_16k", units=64, n=16384, ragged=True),
        # A whole 32-layer cache of 32K tokens, one token: the largest read of memory.
        _case(name="decode_cache_32k", units=256, n=32768, page=128),
        # A layer with an fp32 cache and a sliding window, batch of four, odd group.
        _case(name="decode_window_f32", dtype="f32", units=32, group=3, n=12005, ragged=True,
              page=32, window=4096),
        # A chunk of prefill over a long cache of one layer, every earlier slot visible.
        _case(name="prefill_chunk_16k", tokens=2048, n=16384),
        # Prefill of a layer with a sliding window and sinks.
        _case(name="prefill_window_8k", tokens=8192, n=8192, window=1024),
        # A short fp32 prompt of an odd model: nothing is a multiple of a tile.
        _case(name="prefill_f32_odd", dtype="f32", units=6, group=7, tokens=301, n=1203, page=16),
        # A tree of 64 drafted tokens over the cache of one layer.
        _case(name="tree_layer_8k", op="tree", tokens=64, n=8257),
        # Small trees for a batch of 16 sequences, sliding window, ragged caches.
        _case(name="tree_batch_window", op="tree", units=128, group=5, tokens=13, n=16384,
              ragged=True, page=32, window=2048),
        # A selection over a whole cache, 32K to 2K slots a unit, moved to new pages.
        _case(name="compact_cache_32k", op="compact", units=256, n=32768, keep=2048),
        # Beam search: 4 sequences x 8 beams x 8 KV heads that share their prompts' pages.
        _case(name="beam_step_2k", op="beam", units=256, n=2005, page=16, beams=8),
        # Speculative decoding of a batch of eight, one layer: every cache call of the step.
        _case(name="draft_step_4k", op="draft", units=64, tokens=24, n=4099, page=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case, its sizes spread over the listed ones' range and capped at their work."""
    op = rng.choices(["decode", "prefill", "tree", "compact", "append", "beam", "draft"],
                     [4, 3, 3, 2, 1, 2, 2])[0]
    dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
    page = rng.choice([16, 32, 64, 128])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8])
    window = rng.choice([0, 0, _log_int(rng, 64, 8192)])
    sink = rng.choice([0, 4, rng.randint(1, 200)])
    kw = dict(dtype=dtype, page=page, group=group, window=window, sink=sink,
              ragged=rng.random() < 0.5)
    if op == "decode":
        units = _log_int(rng, 1, 256)
        n = _log_int(rng, 200, min(65536, (8 << 20) // units * (1 if dtype == "bf16" else 0.5)))
        return _case(units=units, n=n, tokens=rng.choice([1, 1, 1, rng.randint(2, 9)]), **kw)
    if op == "prefill":
        units = _log_int(rng, 1, 32)
        most = 2.0e9 if dtype == "bf16" else 2.0e8          # (row, slot) pairs before the mask
        n = _log_int(rng, 100, min(32768, int(math.sqrt(most / units / group))))
        tokens = rng.choice([n, rng.randint(max(1, n // 16), n)])
        return _case(units=units, n=n, tokens=tokens, **dict(kw, ragged=False))
    if op == "tree":
        units = _log_int(rng, 1, 128)
        tokens = rng.choice([rng.randint(2, 64), rng.randint(2, 256)])
        n = _log_int(rng, 16 * tokens + 16, max(16 * tokens + 500, min(32768, (2 << 20) // units)))
        return _case(op="tree", units=units, n=n, tokens=tokens, **kw)
    if op == "compact":
        units = _log_int(rng, 1, 256)
        n = _log_int(rng, 500, min(65536, (8 << 20) // units * (1 if dtype == "bf16" else 0.5)))
        return _case(op="compact", units=units, n=n, keep=_log_int(rng, 20, max(21, n // 8)), **kw)
    if op == "append":
        units = _log_int(rng, 1, 256)
        n = _log_int(rng, 500, min(65536, (4 << 20) // units))
        return _case(op="append", units=units, n=n, tokens=_log_int(rng, 1, n // 16), **kw)
    if op == "beam":
        beams = rng.choice([2, 3, 4, 8])
        units = beams * _log_int(rng, 1, 256 // beams)
        return _case(op="beam", units=units, beams=beams, n=_log_int(rng, 50, 8192),
                     **dict(kw, ragged=False))
    tokens = rng.randint(2, 64)
    return _case(op="draft", units=_log_int(rng, 1, 64), tokens=tokens,
                 n=_log_int(rng, 16 * tokens + 16, 8192), **kw)


# ------------------------------------------------------------------ sizes of a case
def _lens(c):
    """Slots of every unit: n, or spread over [n / 16, n] in a fixed way, the first unit n."""
    if not c["ragged"]:
        return [c["n"]] * c["units"]
    lo = -(-c["n"] // 16)
    return [c["n"] - int((c["n"] - lo) * ((u * 0.6180339887498949) % 1.0))
            for u in range(c["units"])]


def _pages(n, page):
    return -(-n // page)


def _parents(c, gen):
    """Random trees [U][t]: node i hangs on one of the few nodes before it, or on the cache."""
    u, t = c["units"], c["tokens"]
    i = torch.arange(t, device="cuda")
    back = (torch.rand(u, t, device="cuda", generator=gen) ** 2 * 8).long() + 1
    return (i - back).clamp_min(-1).to(torch.int32)


def _depth_of(parent):
    """Depth and ancestor-or-self sets of trees given by parents [U][t], parent < node."""
    t = parent.shape[1]
    node = torch.arange(t, device=parent.device)
    anc = ((node[:, None] == node) | (parent[:, :, None] == node)).float()
    for _ in range((t - 1).bit_length()):       # paths of up to 1, 2, 4 ... steps
        anc = ((anc @ anc) > 0).float()
    anc = anc > 0
    return anc.sum(-1) - 1, anc


def work(case):
    c, es = case, 2 if case["dtype"] == "bf16" else 4
    row = D * es
    lens, t, w, s = _lens(c), c["tokens"], c["window"], c["sink"]
    if c["op"] in ("attend", "tree"):
        rows = c["units"] * c["group"] * t
        slots = pairs = 0
        for n in set(lens):
            base = n - t
            first = max(0, base - w + 1) if w else 0            # first slot of row 0's window
            if c["op"] == "tree":                               # a few of the nodes are seen
                seen = t * (base - first + min(s, first) + 3)
            elif w:
                seen = sum(min(p + 1, w) + min(s, max(0, p + 1 - w)) for p in range(base, n))
            else:
                seen = t * base + t * (t + 1) // 2
            slots += lens.count(n) * (n - first + min(s, first))
            pairs += lens.count(n) * c["group"] * seen
        return {"bytes": slots * 2 * row + rows * (2 * row + 4), "flops": 4 * D * pairs}
    if c["op"] == "compact":
        return {"bytes": c["units"] * c["keep"] * (4 * row + 4), "flops": 0}
    if c["op"] == "append":
        return {"bytes": c["units"] * t * 4 * row, "flops": 0}
    pool = _pool(c)
    table = 4 * sum(_pages(n, c["page"]) for n in lens)
    if c["op"] == "beam":       # tables, counts, the shared part of the last page, one new row
        part = sum(n % c["page"] for n in lens) * 4 * row
        return {"bytes": 4 * table + 8 * pool["pages"] + part + c["units"] * 4 * row, "flops": 0}
    rows = c["units"] * c["group"] * t
    base = sum(n - t for n in lens)
    return {"bytes": 4 * table + 8 * pool["pages"] + c["units"] * t * 4 * row
            + (base + c["units"] * t) * 2 * row + rows * (2 * row + 4),
            "flops": 4 * D * c["group"] * t * base}


def _pool(c):
    """Pages of the pool, columns of the tables, and the first unshared column."""
    lens, page = _lens(c), c["page"]
    cols = _pages(max(lens) + c["tokens"], page) + 1
    if c["op"] == "beam":       # beams of one sequence share the prompt, three quarters
        shared = int(0.75 * c["n"]) // page
        seqs = c["units"] // c["beams"]
        pages = seqs * shared + c["units"] * (cols - shared) * 2
    else:
        shared = 0
        pages = sum(_pages(n, page) for n in lens)
        if c["op"] == "draft":
            pages += c["units"] * (_pages(c["tokens"], page) + 2)
        if c["op"] == "compact":
            pages += c["units"] * _pages(c["keep"], page)
        pages += pages // 16 + 3
    return {"pages": pages, "cols": cols, "shared": shared}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    u, t, page = c["units"], c["tokens"], c["page"]
    lens, pool = _lens(c), _pool(c)
    st = {"case": c, "pool": pool}

    def rnd(*shape, std=1.0, out=torch.float32):
        x = torch.empty(shape, dtype=out, device="cuda")
        flat = x.view(-1)
        for a in range(0, flat.numel(), 1 << 28):
            flat[a:a + (1 << 28)].normal_(0.0, std, generator=g)
        return x

    st["k"], st["v"] = rnd(pool["pages"], page, D, out=dt), rnd(pool["pages"], page, D, out=dt)
    order = torch.randperm(pool["pages"], device="cuda", generator=g).to(torch.int32)
    cols = pool["cols"]
    col = torch.arange(cols, device="cuda")
    len_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    need = (len_d.long() + page - 1) // page
    used = col[None, :] < need[:, None]
    own_col = used & (col[None, :] >= pool["shared"])
    rank = own_col.flatten().long().cumsum(0).view(u, cols) - 1
    head = 0
    table = torch.full((u, cols), -1, dtype=torch.int32, device="cuda")
    if pool["shared"]:
        seqs = u // c["beams"]
        head = seqs * pool["shared"]
        table[:, :pool["shared"]] = order[:head].view(seqs, 1, -1).expand(
            seqs, c["beams"], -1).reshape(u, -1)
    table = torch.where(own_col, order[(rank + head).clamp_min(0)], table)
    st["table"], st["lens"] = table, len_d
    n_used = head + int(own_col.sum())
    # queries share a direction, and the first slots' keys lie along it
    mean = rnd(u, D, std=0.6)
    if c["op"] in ("attend", "tree", "draft") and c["sink"]:
        first = table[:, 0].long()
        k = min(4, c["sink"], page, min(lens))
        st["k"][first, :k] = (2.0 * mean[:, None] + rnd(u, k, D, std=0.3)).to(dt)
    if c["op"] in ("attend", "tree", "draft"):
        st["q"] = (rnd(u, c["group"], t, D, std=1.5) + mean[:, None, None]).to(dt)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(u, c["group"], t, dtype=torch.float32, device="cuda")
    if c["op"] in ("tree", "draft"):
        st["parent"] = _parents(c, g)
    if c["op"] == "compact":
        n = torch.tensor(lens, device="cuda")
        keep = min(c["keep"], min(lens))
        score = torch.rand(u, max(lens), device="cuda", generator=g)
        score[torch.arange(max(lens), device="cuda")[None] >= n[:, None]] = -1
        st["idx"] = score.topk(keep, dim=1).indices.sort(dim=1).values.to(torch.int32)
        st["table_out"] = order[n_used:n_used + u * _pages(keep, page)].view(u, -1)
        pad = torch.full((u, cols - st["table_out"].shape[1]), -1, dtype=torch.int32,
                         device="cuda")
        st["table_out"] = torch.cat([st["table_out"], pad], 1).contiguous()
    if c["op"] == "append":
        st["k_new"], st["v_new"] = rnd(u, t, D, out=dt), rnd(u, t, D, out=dt)
    if c["op"] in ("beam", "draft"):
        st["refs"] = torch.zeros(pool["pages"], dtype=torch.int32, device="cuda")
        st["refs"].index_add_(0, table[used].long(), torch.ones_like(table[used]))
        st["table_b"] = torch.full_like(table, -1)
        st["lens_b"] = torch.zeros_like(len_d)
        st["none"] = torch.zeros_like(len_d)
    if c["op"] == "beam":
        seqs, b = u // c["beams"], c["beams"]
        pick = torch.randint(b, (seqs, b), device="cuda", generator=g)
        st["src"] = (torch.arange(seqs, device="cuda")[:, None] * b + pick).view(-1).to(torch.int32)
        st["want"] = len_d + 1
        st["k_new"], st["v_new"] = rnd(u, 1, D, out=dt), rnd(u, 1, D, out=dt)
    if c["op"] == "draft":
        st["src"] = torch.arange(u, device="cuda", dtype=torch.int32)
        st["want"] = len_d + t
        st["k_new"], st["v_new"] = rnd(u, t, D, out=dt), rnd(u, t, D, out=dt)
        # the accepted path: the ancestors of the deepest node, as verification would give it
        depth, anc = _depth_of(st["parent"])
        deep = depth.argmax(1)
        path = anc[torch.arange(u, device="cuda"), deep]                       # [U][t]
        st["keep"] = path.sum(1).to(torch.int32)
        at = torch.where(path, torch.arange(t, device="cuda"), t + 1).sort(1).values
        st["idx"] = (len_d[:, None] + at.clamp_max(t - 1)).to(torch.int32)
        st["kept_lens"] = len_d + st["keep"]
    if own:
        from paper_2605_31105_gb300 import binding as b
        over = dict(dtype=c["dtype"], window=c["window"], n_sink=c["sink"])

        def plan(tokens):
            return b.cache_params(u, c["group"], pool["pages"], page, cols, tokens=tokens, **over)

        st["p"] = plan(1 if c["op"] == "beam" else keep if c["op"] == "compact" else t)
        st["ws"] = torch.empty(b.grkv_cache_workspace_size(st["p"]), dtype=torch.uint8,
                               device="cuda")
    return st


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    from paper_2605_31105_gb300 import binding as b
    op, p, ws = st["case"]["op"], st["p"], st["ws"]
    if op == "attend":
        b.grkv_attend(p, st["q"], st["k"], st["v"], st["table"], st["lens"], st["out"], ws,
                      lse=st["lse"])
        return st["out"], st["lse"]
    if op == "tree":
        b.grkv_attend_tree(p, st["q"], st["k"], st["v"], st["table"], st["lens"], st["parent"],
                           st["out"], ws, lse=st["lse"])
        return st["out"], st["lse"]
    if op == "compact":
        b.grkv_cache_compact(p, st["idx"], st["k"], st["v"], st["table"], st["lens"],
                             st["table_out"], ws)
        return st["k"], st["v"]
    if op == "append":
        b.grkv_cache_append(p, st["k_new"], st["v_new"], st["k"], st["v"], st["table"],
                            st["lens"], ws)
        return st["k"], st["v"]
    table, lens = st["table_b"], st["lens_b"]
    b.grkv_cache_trim(p, table, st["none"], st["refs"], ws)
    b.grkv_cache_fork(p, st["src"], st["table"], st["lens"], table, lens, st["refs"], ws)
    b.grkv_cache_reserve(p, table, lens, st["want"], st["refs"], st["k"], st["v"], ws)
    b.grkv_cache_append(p, st["k_new"], st["v_new"], st["k"], st["v"], table, st["want"], ws)
    if op == "beam":
        return st["k"], st["v"], table, lens, st["refs"]
    b.grkv_attend_tree(p, st["q"], st["k"], st["v"], table, st["want"], st["parent"],
                       st["out"], ws, lse=st["lse"])
    b.grkv_cache_compact(p, st["idx"], st["k"], st["v"], table, st["want"], table, ws,
                         keep=st["keep"], first=st["lens"])
    b.grkv_cache_trim(p, table, st["kept_lens"], st["refs"], ws)
    return st["k"], st["v"], table, lens, st["refs"], st["out"], st["lse"]


# ------------------------------------------------------------------ the plain forms
def _slots(pages, table, n):
    """Slots 0..n-1 of the given units in fp32, [units][n][D] (entries of no page read page 0)."""
    page = pages.shape[1]
    t = table[:, :_pages(n, page)].long().clamp_min(0)
    return pages[t].float().flatten(1, 2)[:, :n]


def _attend_plain(c, q, k, v, table, lens, n, parent=None):
    u, g, t, _ = q.shape
    w, s, dev = c["window"], c["sink"], q.device
    out = torch.empty_like(q)
    lse = torch.empty(u, g, t, dtype=torch.float32, device=dev)
    j = torch.arange(n, device=dev)
    step = max(1, min(u, (1 << 29) // (n * max(g * t, 2 * D))))
    for a in range(0, u, step):
        z = slice(a, min(u, a + step))
        kk, vv = _slots(k, table[z], n), _slots(v, table[z], n)
        ln = lens[z].long()
        base = (ln - t)[:, None, None]
        i = torch.arange(t, device=dev)[None, :, None]
        if parent is None:
            pos = base + i
            see = j <= pos
            jp = j[None, None]
        else:
            depth, anc = _depth_of(parent[z])
            pos = base + depth[:, :, None]
            node = (j[None] - (ln - t)[:, None]).clamp(0, t - 1)                # [u][n]
            drafted = (j[None] >= (ln - t)[:, None]) & (j[None] < ln[:, None])
            seen = anc.gather(2, node[:, None].expand(-1, t, -1))
            see = torch.where(drafted[:, None], seen, (j[None] < (ln - t)[:, None])[:, None])
            jp = torch.where(drafted, (ln - t)[:, None] + depth.gather(1, node), j[None])[:, None]
        if w:
            see = see & ((jp > pos - w) | (jp < s))
        see = see[:, None]                                                      # [u][1][t][n]
        live = (j[None, :] < ln[:, None])[:, :, None]
        kk, vv = torch.where(live, kk, 0.0), torch.where(live, vv, 0.0)
        x = (q[z].float().flatten(1, 2) @ kk.transpose(1, 2)).view(-1, g, t, n)
        x *= 1.0 / math.sqrt(D)
        x = torch.where(see, x, -math.inf)
        top = x.amax(-1, keepdim=True).clamp_min(-3.0e38)
        x = torch.exp(x - top)
        total = x.sum(-1, keepdim=True)
        o = (x.flatten(1, 2) @ vv).view(-1, g, t, D)
        out[z] = torch.where(total > 0, o / total, 0.0).to(q.dtype)
        lse[z] = (top + torch.log(total))[..., 0]
    return out, lse


def _move(pages, table_in, idx, table_out, dst, live):
    """Slots dst <- slots idx of each unit, where live."""
    page = pages.shape[1]
    rows = torch.arange(idx.shape[0], device=idx.device)[:, None]
    src = table_in[rows, idx // page].long() * page + idx % page
    to = table_out[rows, dst // page].long() * page + dst % page
    flat = pages.view(-1, D)
    flat[to[live]] = flat[src[live]]


def _append_plain(st, table, lens):
    t = st["k_new"].shape[1]
    page = st["k"].shape[1]
    slot = (lens.long() - t)[:, None] + torch.arange(t, device=lens.device)[None]
    at = table.gather(1, slot // page).long() * page + slot % page
    st["k"].view(-1, D)[at.view(-1)] = st["k_new"].view(-1, D)
    st["v"].view(-1, D)[at.view(-1)] = st["v_new"].view(-1, D)


def _add_refs(refs, entries, by):
    ok = entries >= 0
    refs.index_add_(0, entries.clamp_min(0).flatten().long(),
                    (by * ok.to(torch.int32)).flatten())


def _trim_plain(table, lens, refs, page):
    col = torch.arange(table.shape[1], device=table.device)
    drop = col[None] >= ((lens.long() + page - 1) // page)[:, None]
    _add_refs(refs, torch.where(drop, table, -1), -1)
    table.copy_(torch.where(drop, -1, table))


def _fork_plain(st, table, lens):
    page = st["k"].shape[1]
    src = st["src"].long()
    lens.copy_(st["lens"][src])
    col = torch.arange(table.shape[1], device=table.device)
    has = col[None] < ((lens.long() + page - 1) // page)[:, None]
    table.copy_(torch.where(has, st["table"][src], -1))
    _add_refs(st["refs"], table, 1)


def _reserve_plain(st, table, lens, want):
    page, refs = st["k"].shape[1], st["refs"]
    u, cols = table.shape
    col = torch.arange(cols, device=table.device)[None]
    ln, wn = lens.long()[:, None], want.long()[:, None]
    touch = (col >= ln // page) & (col < (wn + page - 1) // page) & (wn > ln)
    held = table >= 0
    shared = held & (refs[table.clamp_min(0).long()] > 1)
    new = touch & (~held | shared)
    free = torch.argsort((refs > 0).to(torch.int32), stable=True)           # free pages first
    rank = new.flatten().long().cumsum(0).view(u, cols) - 1
    fresh = free[rank.clamp_min(0)].to(torch.int32)
    # the filled part of a shared page is copied
    part = (ln[:, 0] % page)
    c0 = (ln[:, 0] // page).clamp_max(cols - 1)
    rows = torch.arange(u, device=table.device)
    copy = new[rows, c0] & (part > 0)
    old, to = table[rows, c0].long().clamp_min(0), fresh[rows, c0].long()
    put = torch.arange(page, device=table.device)[None] < part[:, None]
    put = put & copy[:, None]
    for pool in (st["k"], st["v"]):
        keep = pool[old]
        r, s = put.nonzero(as_tuple=True)
        pool[to[r], s] = keep[r, s]
    _add_refs(refs, torch.where(new & shared, table, -1), -1)
    _add_refs(refs, torch.where(new, fresh, -1), 1)
    table.copy_(torch.where(new, fresh, table))


def _run_plain(st):
    c, op = st["case"], st["case"]["op"]
    page = c["page"]
    if op in ("attend", "tree"):
        return _attend_plain(c, st["q"], st["k"], st["v"], st["table"], st["lens"], c["n"],
                             st.get("parent"))
    if op == "compact":
        idx = st["idx"].long()
        dst = torch.arange(idx.shape[1], device=idx.device)[None].expand_as(idx)
        for pool in (st["k"], st["v"]):
            _move(pool, st["table"], idx, st["table_out"], dst, torch.ones_like(idx).bool())
        return st["k"], st["v"]
    if op == "append":
        _append_plain(st, st["table"], st["lens"])
        return st["k"], st["v"]
    table, lens = st["table_b"], st["lens_b"]
    _trim_plain(table, st["none"], st["refs"], page)
    _fork_plain(st, table, lens)
    _reserve_plain(st, table, lens, st["want"])
    _append_plain(st, table, st["want"])
    if op == "beam":
        return st["k"], st["v"], table, lens, st["refs"]
    out, lse = _attend_plain(c, st["q"], st["k"], st["v"], table, st["want"],
                             c["n"] + c["tokens"], st["parent"])
    idx = st["idx"].long()
    i = torch.arange(idx.shape[1], device=idx.device)[None]
    live = i < st["keep"].long()[:, None]
    for pool in (st["k"], st["v"]):
        _move(pool, table, idx, table, st["lens"].long()[:, None] + i, live)
    _trim_plain(table, st["kept_lens"], st["refs"], page)
    return st["k"], st["v"], table, lens, st["refs"], out, lse


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """The attention outputs, slot by slot of each unit and from the visible set of each row;
    moved rows, tables and counts have no rounding and no value here."""
    c = case
    if c["op"] not in ("attend", "tree", "draft"):
        return None
    pairs = sum(_lens(c)) * c["group"] * c["tokens"]
    if pairs > 8e9:
        return None
    st = prepare(case, seed)
    u, g, t = c["units"], c["group"], c["tokens"]
    lens, page, w, s = _lens(c), c["page"], c["window"], c["sink"]
    out = torch.zeros(u, g, t, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(u, g, t, dtype=torch.float64, device="cuda")
    trees = st["parent"].tolist() if "parent" in st else None
    for x in range(u):
        rows = st["table"][x, :_pages(lens[x], page)].long()
        kk = st["k"][rows].double().reshape(-1, D)[:lens[x]]
        vv = st["v"][rows].double().reshape(-1, D)[:lens[x]]
        if c["op"] == "draft":                       # the drafted rows follow the cache
            kk = torch.cat([kk, st["k_new"][x].double()])
            vv = torch.cat([vv, st["v_new"][x].double()])
        n = kk.shape[0]
        base = n - t
        at = torch.arange(n, device="cuda")          # position of every slot
        if trees is None:
            mine = torch.arange(base, n, device="cuda")
            allowed = None
        else:
            deep, sees = [], torch.zeros(t, t, dtype=torch.bool)
            for i, par in enumerate(trees[x]):
                deep.append(deep[par] + 1 if par >= 0 else 0)
                node = i
                while node >= 0:
                    sees[i, node] = True
                    node = trees[x][node]
            mine = base + torch.tensor(deep, device="cuda")
            at = torch.cat([at[:base], mine])
            allowed = sees.cuda()
        for a in range(0, t, 1024):
            b = min(t, a + 1024)
            ok = at[None, :] <= mine[a:b, None]
            if allowed is not None:
                ok[:, base:] = allowed[a:b]
            if w:
                ok = ok & ((mine[a:b, None] - at[None, :] < w) | (at[None, :] < s))
            for h in range(g):
                logit = st["q"][x, h, a:b].double() @ kk.T / math.sqrt(D)
                logit.masked_fill_(~ok, -math.inf)
                z = torch.logsumexp(logit, 1)
                out[x, h, a:b] = torch.exp(logit - z[:, None]) @ vv
                lse[x, h, a:b] = z
    return (None, None, None, None, None, out, lse) if c["op"] == "draft" else (out, lse)
