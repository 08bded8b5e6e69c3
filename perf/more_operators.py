"""The measured work of positions and encoder states in the paged cache.

A case is one pass through one operator, or, for `stream` and `packed`, through the two calls
that a serving loop makes one after the other.  `op` names it:

  rows     grkv_rope_rows: rotary positions of queries or keys [seqs][heads][tokens][128], or the
           transposed product that a backward pass takes
  append   grkv_cache_append_rope: `tokens` new rows of each unit, keys rotated on their way into the
           pages, and the queries of the same tokens
  packed   the rows of requests of different lengths behind each other: grkv_cache_map makes first
           rows, positions and slots from the lengths, grkv_cache_append_rope takes them
  compact  grkv_cache_compact_rope: kept slots moved to pages of their own, keys turned by what
           their slots change
  stream   a chunk is appended, then half of it evicted in place, keys turned to their new slots
  cross    grkv_attend_cross: queries over encoder states of another length, every slot visible
  map      grkv_cache_map: positions and slots of the new rows of every unit; `tree` gives the
           depths of drafted trees

Sizes: units U = batch x KV heads (x layers), g query heads per KV head, head size 128, `n` slots
of the longest unit with the new rows, `page` slots per page.  `ragged` units hold between n / 16
and n slots, and take between one and `tokens` rows (the same ones for a case).  Pages lie in the
pool in random order.  `offset` is by how much a unit's positions are ahead of its slots, as after
a compression of its prompt.
"""
import math

import torch

own = False

D = 128
_DEFAULTS = dict(op="rows", dtype="bf16", units=8, group=4, tokens=1, n=8192, ragged=False,
                 page=64, keep=0, offset=0, tree=False, rotary=128, layout="half", scaling="plain",
                 theta=10000.0, factor=1.0, original=8192, strided=False, transpose=False)


def _case(**kw):
    return dict(_DEFAULTS, **kw)


def listed():
    return [
        # Queries of one decoding step, 16 sequences of 8 heads at far positions: latency.
        _case(name="rope_step", units=16, group=8, n=131072, theta=500000.0),
        # Queries of a 32K prompt as the projection leaves them, token by token, into the
        # attention's layout: the largest read and write.
        _case(name="rope_prompt_32k", units=1, group=32, tokens=32768, n=32768, theta=500000.0,
              strided=True),
        # A backward pass through interleaved rotations of 50 of 128 dimensions of a long context:
        # fp32, nothing a multiple of a vector.
        _case(name="rope_grad_f32", dtype="f32", units=3, group=7, tokens=1203, n=40001, rotary=50,
              layout="pairs", scaling="yarn", factor=8.0, original=4096, transpose=True),
        # Decoding of a batch of eight, one layer, prompts compressed earlier.
        _case(name="append_step_16k", op="append", units=64, n=16384, ragged=True, offset=100000,
              theta=500000.0, scaling="bands", factor=8.0),
        # A chunk of prefill of one layer, positions past the trained ones.
        _case(name="append_chunk_16k", op="append", tokens=2048, n=16384, scaling="yarn",
              factor=4.0, original=4096),
        # A selection over a whole cache, 32K to 2K slots a unit, keys turned to their new slots.
        _case(name="compact_cache_32k", op="compact", units=256, n=32768, keep=2048,
              theta=500000.0),
        # Streaming with positions of slots: a chunk of 512 appended, half of it evicted in place.
        _case(name="stream_step_4k", op="stream", units=64, tokens=512, n=4099, page=16, keep=256),
        # One token over the encoder states of a batch of 16, as many query as KV heads.
        _case(name="cross_step_1500", op="cross", units=128, group=1, n=1500, ragged=True, page=16),
        # A chunk of a decoder's prompt over long encoder states of one layer: the most operations.
        _case(name="cross_chunk_16k", op="cross", tokens=2048, n=16384),
        # fp32, odd groups and lengths: nothing is a multiple of a tile.
        _case(name="cross_f32_odd", op="cross", dtype="f32", units=6, group=7, tokens=77, n=1203,
              ragged=True, page=16),
        # Positions and slots of a decoding step of 32 sequences of 8 heads.
        _case(name="map_step", op="map", units=256, n=16384, ragged=True, page=16, offset=1000),
        # Positions and slots of 64 drafted nodes in each of 1024 units.
        _case(name="map_tree", op="map", units=1024, tokens=64, n=8192, ragged=True, page=16,
              offset=1000, tree=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case, its sizes spread over the listed ones' range and capped at their work."""
    op = rng.choices(["rows", "append", "packed", "compact", "stream", "cross", "map"],
                     [4, 3, 2, 2, 2, 4, 2])[0]
    dtype = rng.choices(["bf16", "f32"], [3, 2])[0]
    half = 1.0 if dtype == "bf16" else 0.5
    scaling = rng.choice(["plain", "linear", "ntk", "bands", "yarn"])
    kw = dict(op=op, dtype=dtype, page=rng.choice([16, 32, 64, 128]),
              group=rng.choice([1, 2, 3, 4, 5, 7, 8]), ragged=rng.random() < 0.5,
              rotary=rng.choice([128, 128, 64, 2 * rng.randint(1, 64)]),
              layout=rng.choice(["half", "pairs"]), scaling=scaling,
              theta=rng.choice([10000.0, 500000.0]), original=rng.choice([2048, 4096, 8192]),
              factor=1.0 if scaling == "plain" else rng.uniform(1.5, 32.0),
              offset=rng.choice([0, _log_int(rng, 1, 1 << 20)]))
    if op == "rows":
        units, group = _log_int(rng, 1, 64), rng.choice([1, 2, 7, 8, 32, 40])
        tokens = rng.choice([1, _log_int(rng, 1, (1 << 20) // (units * group) * half)])
        return _case(**dict(kw, units=units, group=group, tokens=tokens, ragged=False,
                            n=_log_int(rng, tokens, 1 << 20), strided=rng.random() < 0.5,
                            transpose=rng.random() < 0.4))
    if op in ("append", "packed"):
        units = _log_int(rng, 1, 256)
        n = _log_int(rng, 50, min(32768, (3 << 19) // units * half))
        tokens = _log_int(rng, 1, n // 16)
        return _case(**dict(kw, units=units, n=n, ragged=kw["ragged"] or op == "packed",
                            tokens=rng.choice([1, tokens]) if op == "append" else tokens))
    if op == "compact":
        units = _log_int(rng, 1, 256)
        n = _log_int(rng, 500, min(65536, (8 << 20) // units * half))
        return _case(units=units, n=n, keep=_log_int(rng, 20, n // 16), **kw)
    if op == "stream":
        units = _log_int(rng, 1, 128)
        n = _log_int(rng, 200, min(16384, (1 << 19) // units * half))
        tokens = _log_int(rng, 4, n // 6)
        return _case(**dict(kw, units=units, n=n, tokens=tokens, keep=rng.randint(1, tokens),
                            ragged=False, offset=0))
    if op == "cross":
        units = _log_int(rng, 1, 256)
        tokens = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 2, 2048)])
        pairs = 1.0e9 if dtype == "bf16" else 1.0e8
        most = min(65536, (4 << 20) // units * half, pairs / (units * kw["group"] * tokens))
        return _case(units=units, tokens=tokens, n=_log_int(rng, 1, max(1, int(most))), **kw)
    units, tree = _log_int(rng, 1, 1024), rng.random() < 0.5
    tokens = _log_int(rng, 1, min(256 if tree else 4096, (1 << 17) // units))
    return _case(units=units, tokens=tokens, tree=tree, n=_log_int(rng, 16 * tokens, 65536), **kw)


# ------------------------------------------------------------------ sizes of a case
def _spread(c, lo, hi):
    """A number between lo and hi for every unit, in a fixed way, the first unit's hi."""
    return [hi - int((hi - lo) * ((u * 0.6180339887498949) % 1.0)) for u in range(c["units"])]


def _lens(c):
    return _spread(c, -(-c["n"] // 16), c["n"]) if c["ragged"] else [c["n"]] * c["units"]


def _counts(c):
    """New rows (queries) of every unit: fewer than `tokens` in ragged calls."""
    if not c["ragged"] or c["op"] == "compact":
        return [c["tokens"]] * c["units"]
    return [max(1, min(x, n)) for x, n in zip(_spread(c, 1, c["tokens"]), _lens(c))]


def _pages(n, page):
    return -(-n // page)


def work(case):
    c, es = case, 2 if case["dtype"] == "bf16" else 4
    row, turn = D * es, 3 * case["rotary"]        # six operations for each pair of a row
    lens, rows, g = _lens(c), sum(_counts(c)), c["group"]
    if c["op"] == "rows":
        n = c["units"] * g * c["tokens"]
        return {"bytes": n * 2 * row, "flops": n * turn}
    if c["op"] in ("append", "packed", "stream"):
        b, f = rows * (4 + 2 * g) * row, rows * (1 + g) * turn
        if c["op"] == "stream":
            return {"bytes": b + c["units"] * c["keep"] * (4 * row + 4),
                    "flops": f + c["units"] * c["keep"] * turn}
        return {"bytes": b + (rows * 24 if c["op"] == "packed" else 0), "flops": f}
    if c["op"] == "compact":
        n = c["units"] * c["keep"]
        return {"bytes": n * (4 * row + 4), "flops": n * turn}
    if c["op"] == "cross":
        pairs = sum(a * b for a, b in zip(lens, _counts(c)))
        return {"bytes": sum(lens) * 2 * row + rows * g * (2 * row + 4), "flops": 4 * D * g * pairs}
    cols = sum(_pages(x, c["page"]) + 1 for x in _counts(c))
    return {"bytes": c["units"] * (16 if c["tree"] else 12) + rows * (16 if c["tree"] else 12)
            + 4 * cols, "flops": 0}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _freqs(c):
    """Radians a position of each pair, in 64 bits, and what cosine and sine are multiplied by."""
    r, f, orig = c["rotary"], c["factor"], c["original"]
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    theta = c["theta"]
    if c["scaling"] == "ntk" and r > 2:
        theta = theta * f ** (r / (r - 2))
    freq = theta ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        freq = freq / f
    if c["scaling"] == "bands":                 # 1 and 4 turns over the trained context
        turns = orig * freq / (2 * math.pi)
        keep = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        freq = freq * (keep + (1 - keep) / f)
    if c["scaling"] == "yarn":                  # 1 and 32 turns
        at = [r * math.log(orig / (2 * math.pi * x)) / (2 * math.log(theta)) for x in (32, 1)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        freq = freq * (keep + (1 - keep) / f)
    return freq, 0.1 * math.log(f) + 1 if c["scaling"] == "yarn" and f > 1 else 1.0


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    u, t, page = c["units"], c["tokens"], c["page"]
    lens, counts = _lens(c), _counts(c)
    st = {"case": c, "counts": counts}

    def rnd(*shape, std=1.0, out=dt):
        x = torch.empty(shape, dtype=out, device="cuda")
        flat = x.view(-1)
        for a in range(0, flat.numel(), 1 << 28):
            flat[a:a + (1 << 28)].normal_(0.0, std, generator=g)
        return x

    def ints(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device="cuda")

    st["freq"], st["amp"] = _freqs(c)
    if own:
        from paper_2605_31105_gb300 import binding as b
        st["rope"] = b.grkv_rope_make(b.rope_params(
            rotary=c["rotary"], layout=c["layout"], scaling=c["scaling"], theta=c["theta"],
            factor=c["factor"], original=c["original"]))
    if c["op"] == "rows":
        shape = (u, t, c["group"], D) if c["strided"] else (u, c["group"], t, D)
        x = rnd(*shape)
        st["x"] = x.transpose(1, 2) if c["strided"] else x
        st["out"] = torch.empty(u, c["group"], t, D, dtype=dt, device="cuda")
        start = torch.randint(c["n"] - t + 1, (u,), device="cuda", generator=g)
        st["pos"] = (start[:, None] + torch.arange(t, device="cuda")).to(torch.int32)
        return st

    cols = _pages(max(lens), page) + 1
    need = [_pages(n, page) for n in lens]
    extra = u * _pages(c["keep"], page) if c["op"] == "compact" else 0
    pages = sum(need) + extra + sum(need) // 16 + 3
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    used = torch.arange(cols, device="cuda")[None] < ints(need)[:, None]
    rank = used.flatten().long().cumsum(0).view(u, cols) - 1
    st["table"] = torch.where(used, order[rank.clamp_min(0)], -1)
    st["lens"] = ints(lens)
    st["offset"] = None
    if c["offset"]:
        st["offset"] = torch.randint(c["offset"] + 1, (u,), device="cuda", generator=g,
                                     dtype=torch.int32)
    if c["op"] != "map":
        st["k"], st["v"] = rnd(pages, page, D), rnd(pages, page, D)
    st["count"] = ints(counts) if c["ragged"] else None
    if c["op"] in ("append", "packed", "stream"):
        rows = (sum(counts),) if c["op"] == "packed" else (u, t)
        st["k_new"], st["v_new"] = rnd(*rows, D), rnd(*rows, D)
        st["q"] = rnd(u, c["group"], t, D, std=1.5)
        st["q_out"] = torch.zeros_like(st["q"])
    if c["op"] in ("packed", "map"):
        st["pos"] = torch.empty(u, t, dtype=torch.int32, device="cuda")
        st["slot"] = torch.empty(u, t, dtype=torch.int64, device="cuda")
        st["first_row"] = None
        if c["op"] == "packed":
            st["first_row"] = torch.empty(u + 1, dtype=torch.int64, device="cuda")
    st["parent"] = None
    if c["tree"]:
        i = torch.arange(t, device="cuda")
        back = (torch.rand(u, t, device="cuda", generator=g) ** 2 * 8).long() + 1
        st["parent"] = (i - back).clamp_min(-1).to(torch.int32)
    keep = c["keep"]
    if c["op"] == "compact":
        keep = min(keep, min(lens))
        score = torch.rand(u, max(lens), device="cuda", generator=g)
        score[torch.arange(max(lens), device="cuda")[None] >= st["lens"][:, None]] = -1
        st["idx"] = score.topk(keep, dim=1).indices.sort(dim=1).values.to(torch.int32)
        out = order[sum(need):sum(need) + u * _pages(keep, page)].view(u, -1)
        st["table_out"] = torch.full_like(st["table"], -1)
        st["table_out"][:, :out.shape[1]] = out
    if c["op"] == "stream":          # kept rows of the chunk, in place, from the chunk's first slot
        score = torch.rand(u, t, device="cuda", generator=g)
        kept = score.topk(keep, dim=1).indices.sort(dim=1).values
        st["first"] = st["lens"] - t
        st["idx"] = (st["first"][:, None] + kept).to(torch.int32)
    if c["op"] == "cross":
        st["q"] = rnd(u, c["group"], t, D, std=1.5)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(u, c["group"], t, dtype=torch.float32, device="cuda")
    if own:
        def plan(tokens):
            return b.cache_params(u, c["group"], pages, page, cols, tokens=tokens,
                                  dtype=c["dtype"])

        st["p"] = plan(keep if c["op"] == "compact" else t)
        st["p_keep"] = plan(keep) if c["op"] == "stream" else None
        st["ws"] = torch.empty(max(b.grkv_cache_workspace_size(p) for p in
                                   (st["p"], st["p_keep"]) if p), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    from paper_2605_31105_gb300 import binding as b
    c, op = st["case"], st["case"]["op"]
    if op == "rows":
        b.grkv_rope_rows(st["rope"], st["x"], st["out"], pos=st["pos"], transpose=c["transpose"])
        return st["out"]
    p, ws = st["p"], st["ws"]
    if op == "cross":
        b.grkv_attend_cross(p, st["q"], st["k"], st["v"], st["table"], st["lens"], st["out"], ws,
                            q_lens=st["count"], lse=st["lse"])
        return st["out"], st["lse"]
    if op == "compact":
        b.grkv_cache_compact_rope(p, st["rope"], st["idx"], st["k"], st["v"], st["table"],
                                  st["lens"], st["table_out"], ws)
        return st["k"], st["v"]
    if op in ("map", "packed"):
        b.grkv_cache_map(p, st["table"], st["lens"], st["pos"], st["slot"], ws,
                         count=st["count"], parent=st["parent"], offset=st["offset"],
                         first_row=st["first_row"])
        if op == "map":
            return st["pos"], st["slot"]
        b.grkv_cache_append_rope(p, st["rope"], st["k_new"], st["v_new"], st["k"], st["v"],
                                 st["table"], st["lens"], ws, q=st["q"], q_out=st["q_out"],
                                 pos=st["pos"], count=st["count"], first_row=st["first_row"])
        return st["k"], st["v"], st["q_out"], st["pos"], st["slot"], st["first_row"]
    b.grkv_cache_append_rope(p, st["rope"], st["k_new"], st["v_new"], st["k"], st["v"],
                             st["table"], st["lens"], ws, q=st["q"], q_out=st["q_out"],
                             offset=st["offset"], count=st["count"])
    if op == "stream":
        b.grkv_cache_compact_rope(st["p_keep"], st["rope"], st["idx"], st["k"], st["v"],
                                  st["table"], st["lens"], st["table"], ws, first=st["first"])
    return st["k"], st["v"], st["q_out"]


# ------------------------------------------------------------------ the plain forms
def _turned(c, x, pos, freq, amp, transpose=False):
    """Rows x [..., D] rotated to positions pos [...], in 32 bits with angles in 64."""
    r = c["rotary"]
    ang = pos.double()[..., None] * freq
    cos, sin = (torch.cos(ang) * amp).float(), (torch.sin(ang) * amp).float()
    if transpose:
        sin = -sin
    out = x.float()
    if c["layout"] == "half":
        a, b = out[..., :r // 2], out[..., r // 2:r]
    else:
        a, b = out[..., 0:r:2], out[..., 1:r:2]
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.cat([a, b], -1) if c["layout"] == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([y, out[..., r:]], -1).to(x.dtype)


def _live(st, t):
    i = torch.arange(t, device="cuda")[None]
    return i < (torch.full_like(st["lens"], t) if st["count"] is None else st["count"])[:, None]


def _map_plain(st):
    """Slot, position and row of the pool of every new row [U][t]; -1 where there is none."""
    c = st["case"]
    t, page = c["tokens"], c["page"]
    live = _live(st, t)
    i = torch.arange(t, device="cuda")[None]
    base = st["lens"].long() - live.sum(1)
    slot = base[:, None] + i
    pos = slot
    if st["parent"] is not None:
        node = torch.arange(t, device="cuda")
        anc = ((node[:, None] == node) | (st["parent"][:, :, None] == node)).float()
        for _ in range((t - 1).bit_length()):
            anc = ((anc @ anc) > 0).float()
        pos = base[:, None] + anc.sum(-1).long() - 1
    if st["offset"] is not None:
        pos = pos + st["offset"].long()[:, None]
    at = st["table"].gather(1, slot.clamp_min(0) // page).long() * page + slot % page
    return live, torch.where(live, pos, -1), torch.where(live, at, -1)


def _append_plain(st, live, pos, at):
    """pos, at [U][t]; new rows by unit, or packed."""
    c = st["case"]
    new = pos[live] if st["k_new"].dim() == 2 else pos
    k = _turned(c, st["k_new"], new, st["freq"], st["amp"])
    pick = (lambda x: x) if st["k_new"].dim() == 2 else (lambda x: x[live])
    st["k"].view(-1, D)[at[live]] = pick(k)
    st["v"].view(-1, D)[at[live]] = pick(st["v_new"])
    q = _turned(c, st["q"], pos[:, None], st["freq"], st["amp"])
    st["q_out"].copy_(torch.where(live[:, None, :, None], q, st["q_out"]))


def _compact_plain(st, table_out, first):
    c = st["case"]
    page, idx = c["page"], st["idx"].long()
    rows = torch.arange(idx.shape[0], device="cuda")[:, None]
    dst = first.long()[:, None] + torch.arange(idx.shape[1], device="cuda")[None]
    src = st["table"][rows, idx // page].long() * page + idx % page
    to = table_out[rows, dst // page].long() * page + dst % page
    k, v = st["k"].view(-1, D), st["v"].view(-1, D)
    k[to.flatten()] = _turned(c, k[src.flatten()], (dst - idx).flatten(), st["freq"], 1.0)
    v[to.flatten()] = v[src.flatten()]


def _cross_plain(st):
    c, q, lens, n = st["case"], st["q"], st["lens"], st["case"]["n"]
    u, g, t, _ = q.shape
    page = c["page"]
    live = _live(st, t)
    step = max(1, min(u, (1 << 29) // (n * max(g * t, 2 * D))))
    j = torch.arange(n, device="cuda")
    for a in range(0, u, step):
        z = slice(a, min(u, a + step))
        tab = st["table"][z, :_pages(n, page)].long().clamp_min(0)
        has = j[None] < lens[z, None]
        kk, vv = (torch.where(has[..., None], x[tab].flatten(1, 2)[:, :n].float(), 0.0)
                  for x in (st["k"], st["v"]))
        x = q[z].float().flatten(1, 2) @ kk.transpose(1, 2) * (1.0 / math.sqrt(D))
        x = torch.where(has[:, None], x, -math.inf)
        top = x.amax(-1, keepdim=True).clamp_min(-3.0e38)
        x = torch.exp(x - top)
        total = x.sum(-1, keepdim=True)
        o = torch.where(total > 0, (x @ vv) / total, 0.0).view(-1, g, t, D)
        lse = (top + torch.log(total)).view(-1, g, t)
        st["out"][z] = torch.where(live[z, None, :, None], o.to(q.dtype), st["out"][z])
        st["lse"][z] = torch.where(live[z, None], lse, st["lse"][z])
    return st["out"], st["lse"]


def _run_plain(st):
    c, op = st["case"], st["case"]["op"]
    if op == "rows":
        st["out"].copy_(_turned(c, st["x"], st["pos"][:, None], st["freq"], st["amp"],
                                c["transpose"]))
        return st["out"]
    if op == "cross":
        return _cross_plain(st)
    if op == "compact":
        _compact_plain(st, st["table_out"], torch.zeros_like(st["lens"]))
        return st["k"], st["v"]
    live, pos, at = _map_plain(st)
    if op == "map":
        st["pos"].copy_(pos)
        st["slot"].copy_(at)
        return st["pos"], st["slot"]
    if op == "packed":
        n = int(sum(st["counts"]))
        for to, x in ((st["pos"], pos), (st["slot"], at)):
            to.fill_(-1)
            to.view(-1)[:n] = x[live].to(to.dtype)
        st["first_row"].zero_()
        st["first_row"][1:] = live.sum(1).cumsum(0)
    _append_plain(st, live, pos, at)
    if op == "packed":
        return st["k"], st["v"], st["q_out"], st["pos"], st["slot"], st["first_row"]
    if op == "stream":
        _compact_plain(st, st["table"], st["first"])
    return st["k"], st["v"], st["q_out"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_freq(c, i):
    """Radians a position of pair i, number by number."""
    r, f, o = c["rotary"], c["factor"], c["original"]
    plain = math.exp(-2.0 * i / r * math.log(c["theta"]))
    if c["scaling"] == "linear":
        return plain / f
    if c["scaling"] == "ntk":
        return plain * (f ** (-2.0 * i / (r - 2)) if r > 2 else 1.0)
    if c["scaling"] == "bands":
        length = 2 * math.pi / plain
        if length < o / 4:
            return plain
        if length > o:
            return plain / f
        s = (o / length - 1) / 3
        return (1 - s) * plain / f + s * plain
    if c["scaling"] == "yarn":
        where = lambda x: r * math.log(o / (x * 2 * math.pi)) / (2 * math.log(c["theta"]))
        lo, hi = max(math.floor(where(32)), 0), min(math.ceil(where(1)), r - 1)
        ramp = min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
        return plain / f * ramp + plain * (1 - ramp)
    return plain


def _exact_turned(c, x, pos, amp, sign=1):
    """Pairs as complex numbers times amp exp(+-i angle)."""
    r = c["rotary"]
    out = x.double().clone()
    for i in range(r // 2):
        a, b = (i, i + r // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        ang = pos.double() * (sign * _exact_freq(c, i))
        z = torch.complex(out[..., a], out[..., b]) * torch.polar(torch.full_like(ang, amp), ang)
        out[..., a], out[..., b] = z.real, z.imag
    return out


def exact(case, seed):
    """Rotated rows and attention outputs; values that are only moved, tables, positions and slots
    have no rounding and no value here."""
    c = case
    if c["op"] == "map":
        return None
    st = prepare(case, seed)
    u, t, page = c["units"], c["tokens"], c["page"]
    amp = 0.1 * math.log(c["factor"]) + 1 if c["scaling"] == "yarn" and c["factor"] > 1 else 1.0
    if c["op"] == "rows":
        return _exact_turned(c, st["x"], st["pos"][:, None], amp, -1 if c["transpose"] else 1)
    lens, counts = _lens(c), _counts(c)
    if c["op"] == "cross":
        if sum(lens) * c["group"] * t > 8e9:
            return None
        out = torch.zeros(u, c["group"], t, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(u, c["group"], t, dtype=torch.float64, device="cuda")
        for x in range(u):
            rows = st["table"][x, :_pages(lens[x], page)].long()
            kk = st["k"][rows].double().reshape(-1, D)[:lens[x]]
            vv = st["v"][rows].double().reshape(-1, D)[:lens[x]]
            for h in range(c["group"]):
                logit = st["q"][x, h, :counts[x]].double() @ kk.T / math.sqrt(D)
                z = torch.logsumexp(logit, 1)
                out[x, h, :counts[x]] = torch.exp(logit - z[:, None]) @ vv
                lse[x, h, :counts[x]] = z
        return out, lse
    k = st["k"].double()
    flat = k.view(-1, D)

    def rows_of(x, slots, table):
        return table[x].long()[slots // page] * page + slots % page

    if c["op"] == "compact":
        for x in range(u):
            idx = st["idx"][x].long()
            to = torch.arange(idx.shape[0], device="cuda")
            flat[rows_of(x, to, st["table_out"])] = _exact_turned(
                c, st["k"].view(-1, D)[rows_of(x, idx, st["table"])], to - idx, 1.0)
        return k, None
    q = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    ahead = [0] * u if st["offset"] is None else st["offset"].tolist()
    row = 0
    for x in range(u):
        m = counts[x]
        slots = torch.arange(lens[x] - m, lens[x], device="cuda")
        new = st["k_new"][row:row + m] if c["op"] == "packed" else st["k_new"][x, :m]
        row += m
        turned = _exact_turned(c, new, slots + ahead[x], amp)
        if c["op"] == "stream":      # rounded once where it is appended, then moved and turned
            turned = turned.to(st["k"].dtype).double()
        flat[rows_of(x, slots, st["table"])] = turned
        q[x, :, :m] = _exact_turned(c, st["q"][x, :, :m], (slots + ahead[x])[None], amp)
        if c["op"] == "stream":
            idx = st["idx"][x].long()
            to = lens[x] - t + torch.arange(idx.shape[0], device="cuda")
            flat[rows_of(x, to, st["table"])] = _exact_turned(
                c, flat[rows_of(x, idx, st["table"])].clone(), to - idx, 1.0)
    return (k, None, q, None, None, None) if c["op"] == "packed" else (k, None, q)
