"""Performance cases of the paged cache: the target model answers from its translated context.

Four operators over one cache (pools of pages for every layer's keys and values, a page table, lengths):
``paged_attention`` (a chunk of new tokens, one to thousands, over the cache), ``cache_append`` (norms of queries and
keys, position rotation, keys and values stored into their pages; without norms and rotation a translated cache of all
layers is stored), ``cache_reorder`` (rows of the table take prefixes of other rows: forks, copies, truncation, freed
and added pages) and ``cache_compact`` (the pages in use move to the lowest numbers).

Head layouts are those of the models in ``paper_2607_28979_amd.configs`` and the replay cases. Lengths, parents and
forks go by the case; values and the places of pages by the seed.
"""
import math
import random

import torch

own = False

#: (query heads, KV heads, head dim, type)
HEADS = {"q7b": (28, 4, 128, "bf16"), "q1.5b": (12, 2, 128, "bf16"), "q0.5b": (14, 2, 64, "bf16"),
         "mha64": (16, 16, 64, "bf16"), "opt125m": (12, 12, 64, "f32"), "q1.5b_f32": (12, 2, 128, "f32")}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ROPE_BASE, EPS = 1e6, 1e-6


def listed():
    return [
        # one decoded token of one conversation on a short context: latency
        _attend("decode_1_ctx1100", "q7b", B=1, new=1, ctx=1100, page=16),
        # a decode step of a serving batch whose contexts differ widely: cache bandwidth
        _attend("decode_48_ragged8k", "q7b", B=48, new=1, ctx=8192, page=64, ragged=True),
        # a short turn of several conversations, packed, pages in head-major layout
        _attend("turn_6x37_ctx4k", "q1.5b", B=6, new=37, ctx=4096, page=32, layout=1, ragged=True),
        # a chunk of a long prompt over the context before it: matrix work
        _attend("prompt_2x2048_ctx8k", "q7b", B=2, new=2048, ctx=8192, page=64),
        # the smallest configuration, fp32 caches
        _attend("prompt_f32_3x64_ctx333", "opt125m", B=3, new=64, ctx=333, page=16, ragged=True),
        # a decode step's new keys and values, rotated (and normed), one layer
        _append("append_32x1", "q7b", B=32, new=1, ctx=4096, page=64, norm=True),
        # a prompt chunk's rows, rotation only
        _append("append_1x4096", "q7b", B=1, new=4096, ctx=8000, page=64),
        # a translated context of every layer put into pages (head-major rows, an odd length)
        _append("store_28x1501", "q7b", B=1, new=1501, ctx=1501, page=16, L=28, plain=True, rows="bhtd"),
        # a beam search step: every row takes a parent of its group of eight, all layers
        _reorder("beams_64", "q1.5b", B=64, ctx=1500, page=32, L=28, beams=8),
        # upkeep of a serving batch: rows grow, some fork, some end and make room
        _reorder("upkeep_200", "q0.5b", B=200, ctx=2000, page=16, L=24, beams=1),
        # a small pool squeezed together after half of its sequences ended
        _compact("squeeze_12", "q0.5b", B=12, ctx=300, page=16, L=24),
        # a larger pool
        _compact("squeeze_96", "q7b", B=96, ctx=1800, page=32, L=14, layout=1),
    ]


def _attend(name, heads, B, new, ctx, page, layout=0, ragged=False, window=0):
    return {"name": name, "op": "attend", "heads": heads, "B": B, "new": new, "ctx": ctx, "page": page,
            "layout": layout, "ragged": ragged, "window": window}


def _append(name, heads, B, new, ctx, page, layout=0, ragged=False, L=1, norm=False, plain=False, rows="bthd",
            inter=False):
    return {"name": name, "op": "append", "heads": heads, "B": B, "new": new, "ctx": ctx, "page": page,
            "layout": layout, "ragged": ragged, "L": L, "norm": norm, "plain": plain, "rows": rows, "inter": inter}


def _reorder(name, heads, B, ctx, page, L, beams, layout=0):
    return {"name": name, "op": "reorder", "heads": heads, "B": B, "ctx": ctx, "page": page, "L": L, "beams": beams,
            "layout": layout}


def _compact(name, heads, B, ctx, page, L, layout=0):
    return {"name": name, "op": "compact", "heads": heads, "B": B, "ctx": ctx, "page": page, "L": L, "layout": layout}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend"] * 6 + ["append"] * 3 + ["reorder"] * 2 + ["compact"] * 2)
    c = {"page": rng.choice([16, 16, 32, 64, 128]), "layout": rng.choice([0, 0, 1])}
    if op == "attend":
        heads = rng.choice(["q7b", "q7b", "q1.5b", "q0.5b", "mha64", "opt125m", "q1.5b_f32"])
        if rng.random() < 0.5:   # decoding
            B = _log_int(rng, 1, 64)
            new, ctx = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 64, 32768 if B < 12 else 8192)
        else:                    # chunks of a prompt
            B, new = rng.choice([1, 1, 2, 5]), _log_int(rng, 7, 1024)
            ctx = new + _log_int(rng, 1, 4096)
        c.update(_attend("", heads, B, new, ctx, c["page"], c["layout"], ragged=rng.random() < 0.6,
                         window=rng.choice([0, 0, 0, 500, 1024])))
    elif op == "append":
        heads = rng.choice(list(HEADS))
        plain = rng.random() < 0.3
        B, new = _log_int(rng, 1, 32), _log_int(rng, 1, 4096)
        new = max(1, min(new, 4096 // B))
        c.update(_append("", heads, B, new, new + _log_int(rng, 1, 8192 // B), c["page"], c["layout"],
                         ragged=rng.random() < 0.5, L=rng.choice([1, 4, 12]) if plain else 1, norm=rng.random() < 0.5,
                         plain=plain, rows=rng.choice(["bthd", "bhtd"]), inter=rng.random() < 0.3))
        if c["ragged"]:
            c["rows"] = "bthd"
    else:
        heads = rng.choice(["q7b", "q1.5b", "q0.5b", "opt125m"])
        L = rng.choice([1, 6, 12, 24])
        most = 1 << 29                                    # bytes of a pool
        _, h, d, t = HEADS[heads]
        B = _log_int(rng, 2, 200)
        ctx = _log_int(rng, 40, max(41, min(4000, most // (L * B * h * d * (4 if t == "f32" else 2)))))
        if op == "reorder":
            c.update(_reorder("", heads, B, ctx, c["page"], L, rng.choice([1, 1, 2, 4, 8]), c["layout"]))
        else:
            c.update(_compact("", heads, B, ctx, c["page"], L, c["layout"]))
    del c["name"]
    return c


# what goes by the case alone ------------------------------------------------------------------------------------------

def _rng(c):
    return random.Random("%s %d %d %d" % (c["op"], c["B"], c["ctx"], c["page"]))


def _lengths(c):
    """(kv lengths with the new tokens, new tokens) of every sequence. Ragged: contexts and turns differ."""
    B, new, ctx = c["B"], c["new"], c["ctx"]
    if not c["ragged"]:
        return [ctx - (b * 3) % (1 + (ctx - new) // 8) for b in range(B)], [new] * B
    r = _rng(c)
    n = [new if b == 0 else max(1, round(new * r.uniform(0.1, 1.0))) for b in range(B)]
    lens = [ctx if b == 0 else max(n[b], _log_int(r, max(1, ctx // 40), ctx)) for b in range(B)]
    return lens, n


def _parents(c):
    """(old lengths, source row, kept positions, wanted positions) of a reordering of B rows."""
    r, B, ctx = _rng(c), c["B"], c["ctx"]
    if c["beams"] > 1:
        group = [_log_int(r, max(2, ctx // 4), ctx) for _ in range(-(-B // c["beams"]))]
        old = [group[b // c["beams"]] for b in range(B)]
        src = [min(B - 1, b - b % c["beams"] + r.randrange(c["beams"])) for b in range(B)]
        src = [s if s // c["beams"] == b // c["beams"] else b for b, s in enumerate(src)]
        keep = [old[s] for s in src]
        return old, src, keep, [k + 1 for k in keep]
    old = [_log_int(r, max(2, ctx // 40), ctx) for _ in range(B)]
    src, keep, want = [], [], []
    for b in range(B):
        x = r.random()
        if x < 0.8:         # goes on
            s, k, w = b, old[b], old[b] + 1
        elif x < 0.88:      # forked from another row
            s = r.randrange(B)
            k, w = old[s], old[s] + 1
        elif x < 0.94:      # cut back
            s, k = b, r.randrange(old[b])
            w = k + 1
        else:               # ended; a new prompt takes the row
            s, k, w = -1, 0, _log_int(r, 1, ctx)
        src.append(s)
        keep.append(k)
        want.append(w)
    return old, src, keep, want


def _alive(c):
    """Lengths of the rows that a compaction keeps; 0: the row ended and its pages lie free among the others'."""
    r = _rng(c)
    lens = [_log_int(r, max(1, c["ctx"] // 10), c["ctx"]) for _ in range(c["B"])]
    return lens, [n if r.random() < 0.6 else 0 for n in lens]


def _pages(n, ps):
    return -(-n // ps)


# inputs ---------------------------------------------------------------------------------------------------------------

class _Draw:
    """Seeded random tensors on the GPU, rounded to the storage type."""

    def __init__(self, seed, dtype):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.dtype = dtype

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").to(self.dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.gen, device="cuda").int()


def _ints(v):
    return torch.tensor(v, device="cuda", dtype=torch.int32)


def _pool(g, c, L, n_pages):
    _, h, d, _ = HEADS[c["heads"]]
    shape = (c["page"], h) if not c["layout"] else (h, c["page"])
    out = torch.empty((L, n_pages, *shape, d), device="cuda", dtype=g.dtype)
    for layer in out:
        layer.copy_(g.normal(n_pages, *shape, d))
    return out


def _table(g, counts, cols, n_pages):
    """Rows of `counts` pages each, at places of the pool in random order; -1 past them."""
    t = torch.full((len(counts), cols), -1, device="cuda", dtype=torch.int32)
    at = torch.arange(cols, device="cuda")[None, :] < torch.tensor(counts, device="cuda")[:, None]
    t[at] = g.order(n_pages)[:sum(counts)]
    return t


def prepare(case, seed):
    c = case
    hq, h, d, t = HEADS[c["heads"]]
    g, ps, B = _Draw(seed, TYPES[t]), c["page"], c["B"]
    s = {"case": c}
    if c["op"] in ("attend", "append"):
        lens, n = _lengths(c)
        counts = [_pages(x, ps) for x in lens]
        n_pages = sum(counts) + 3
        L = c.get("L", 1)
        s.update(k_pages=_pool(g, c, L, n_pages), v_pages=_pool(g, c, L, n_pages),
                 table=_table(g, counts, max(counts) + 1, n_pages), kv_len=_ints(lens), max_new=max(n), start=None)
        if c["ragged"]:
            s["start"] = _ints([sum(n[:b]) for b in range(B + 1)])
        rows = (sum(n),) if c["ragged"] else (B, c["new"])

        def new(heads, L=None):
            if c.get("rows") == "bhtd":
                return g.normal(*(() if L is None else (L,)), B, heads, c["new"], d).transpose(-3, -2)
            return g.normal(*(() if L is None else (L,)), *rows, heads, d)

        if c["op"] == "attend":
            s["k_pages"], s["v_pages"] = s["k_pages"][0], s["v_pages"][0]
            s["q"] = new(hq)
            s["o"] = torch.zeros_like(s["q"])
        else:
            s["k"], s["v"] = new(h, L), new(h, L)
            s["q"] = s["q_out"] = s["q_gain"] = s["k_gain"] = s["inv_freq"] = None
            if not c["plain"]:
                s["q"] = new(hq, L)
                s["q_out"] = torch.zeros((L, *rows, hq, d), device="cuda", dtype=g.dtype)
                i = torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d
                s["inv_freq"] = (ROPE_BASE ** -i).float()
                if c["norm"]:
                    s["q_gain"], s["k_gain"] = (1 + 0.1 * g.normal(L, d) for _ in range(2))
    elif c["op"] == "reorder":
        old, src, keep, want = _parents(c)
        counts = [_pages(x, ps) for x in old]
        n_pages = sum(counts) + sum(_pages(x, ps) for x in want) // 4 + B
        s.update(k_pages=_pool(g, c, c["L"], n_pages), v_pages=_pool(g, c, c["L"], n_pages),
                 table=_table(g, counts, _pages(max(old + want), ps), n_pages), source=_ints(src), keep=_ints(keep),
                 want=_ints(want), missing=_ints([0]))
        s["new_table"] = torch.zeros_like(s["table"])
    else:
        lens, alive = _alive(c)
        counts = [_pages(x, ps) for x in lens]
        n_pages = sum(counts) + 3
        table = _table(g, counts, max(counts), n_pages)
        table[_ints(alive) == 0] = -1
        s.update(k_pages=_pool(g, c, c["L"], n_pages), v_pages=_pool(g, c, c["L"], n_pages), table=table,
                 new_table=torch.zeros_like(table), used=_ints([0]))
    return s


# one pass -------------------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": _own_attend, "append": _own_append, "reorder": _own_reorder, "compact": _own_compact}[op](s)
    return {"attend": _attend32, "append": _append32, "reorder": _reorder32, "compact": _compact32}[op](s)


def _own_attend(s):
    from paper_2607_28979_amd import binding as mb
    mb.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["o"], new_start=s["start"],
                       max_new=s["max_new"], window=s["case"]["window"], page_layout=s["case"]["layout"])
    return {"o": s["o"]}


def _own_append(s):
    from paper_2607_28979_amd import binding as mb
    mb.cache_append(s["q"], s["k"], s["v"], s["q_out"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"],
                    new_start=s["start"], max_new=s["max_new"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS,
                    inv_freq=s["inv_freq"], interleaved=s["case"]["inter"], page_layout=s["case"]["layout"])
    return {"k": s["k_pages"], "v": s["v_pages"], **({} if s["q"] is None else {"q": s["q_out"]})}


def _own_reorder(s):
    from paper_2607_28979_amd import binding as mb
    mb.cache_reorder(s["k_pages"], s["v_pages"], s["table"], s["source"], s["keep"], s["want"], s["new_table"],
                     s["missing"], page_layout=s["case"]["layout"])
    return {"k": s["k_pages"], "v": s["v_pages"], "table": s["new_table"], "missing": s["missing"]}


def _own_compact(s):
    from paper_2607_28979_amd import binding as mb
    mb.cache_compact(s["k_pages"], s["v_pages"], s["table"], s["new_table"], s["used"],
                     page_layout=s["case"]["layout"])
    return {"k": s["k_pages"], "v": s["v_pages"], "table": s["new_table"], "used": s["used"]}


# the plain forms ------------------------------------------------------------------------------------------------------

def _new_rows(s, rows_each):
    """(sequence, row among the rows of all sequences, position) of every new token."""
    B, dev = s["table"].shape[0], s["table"].device
    if s["start"] is None:
        b = torch.arange(B, device=dev).repeat_interleave(rows_each)
        row = torch.arange(B * rows_each, device=dev)
        i = row - b * rows_each
        n = torch.full((B,), rows_each, device=dev)
    else:
        n = (s["start"][1:] - s["start"][:-1]).long()
        b = torch.arange(B, device=dev).repeat_interleave(n)
        row = torch.arange(b.shape[0], device=dev)
        i = row - s["start"].long()[b]
    return b, row, s["kv_len"].long()[b] - n[b] + i


def _attend32(s):
    c, (hq, h, d, _) = s["case"], HEADS[s["case"]["heads"]]
    B, ps, mn, G = c["B"], c["page"], s["max_new"], hq // h
    q, o = s["q"].view(-1, hq, d), s["o"].view(-1, hq, d)
    if s["start"] is None:
        b = i = None
        qb = q.view(B, mn, hq, d).float()
        n = torch.full((B,), mn, device=q.device)
    else:
        n = (s["start"][1:] - s["start"][:-1]).long()
        i, b = torch.arange(mn, device=q.device), torch.arange(B, device=q.device)
        there = i[None] < n[:, None]
        rows = (s["start"][:-1].long()[:, None] + i[None]).clamp(max=q.shape[0] - 1)
        qb = q[rows].float()
    kv = s["kv_len"].long()
    pages = s["table"].long()
    good = (pages >= 0) & (pages < s["k_pages"].shape[0])
    pos = torch.arange(pages.shape[1] * ps, device=q.device)

    def cache(pool):
        x = pool[pages.clamp(0, pool.shape[0] - 1)]
        x = x.transpose(2, 3) if c["layout"] else x
        x = x.reshape(B, -1, h, d)
        x = torch.where(held[:, :, None, None], x, torch.zeros((), device=x.device, dtype=x.dtype))
        return x.float().permute(0, 2, 1, 3).contiguous()          # [B][h][position][d]

    held = good.repeat_interleave(ps, 1) & (pos[None] < kv[:, None])
    at = kv[:, None] - n[:, None] + torch.arange(mn, device=q.device)[None]    # [B][new]
    see = held[:, None] & (pos[None, None] <= at[:, :, None])
    if c["window"]:
        see &= pos[None, None] > at[:, :, None] - c["window"]
    qh = qb.view(B, mn, h, G, d).permute(0, 2, 3, 1, 4).reshape(B, h, G * mn, d)
    sc = torch.matmul(qh, cache(s["k_pages"]).transpose(2, 3).contiguous()).view(B, h, G, mn, -1)
    sc = sc.mul_(1 / math.sqrt(d)).masked_fill_(~see[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = sc.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, h, G * mn, -1), cache(s["v_pages"])).view(B, h, G, mn, d)
    out = (out / total.clamp(min=1e-30)).permute(0, 3, 1, 2, 4).reshape(B, mn, hq, d).to(o.dtype)
    if s["start"] is None:
        o.copy_(out.reshape(-1, hq, d))
    else:
        o[rows[there]] = out[there]
    return {"o": s["o"]}


def _rotate32(x, angle_cos, angle_sin, inter):
    half = x.shape[-1] // 2
    a, b = (x[..., 0::2], x[..., 1::2]) if inter else (x[..., :half], x[..., half:])
    u, v = a * angle_cos - b * angle_sin, b * angle_cos + a * angle_sin
    return torch.stack((u, v), -1).flatten(-2) if inter else torch.cat((u, v), -1)


def _append32(s):
    c = s["case"]
    ps, rows_each = c["page"], c["new"]
    b, row, pos = _new_rows(s, rows_each)
    page = s["table"].long()[b, (pos.clamp(min=0) // ps)]
    slot = pos.clamp(min=0) % ps
    flat = lambda x: x.reshape(x.shape[0], -1, *x.shape[-2:])       # noqa: E731
    if s["inv_freq"] is not None:
        angle = pos.double()[:, None] * s["inv_freq"].double()[None]
        cos, sin = angle.cos().float()[None, :, None], angle.sin().float()[None, :, None]

    def ready(x, gain):
        if s["inv_freq"] is None and gain is None:
            return flat(x)
        y = flat(x).float()
        if gain is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gain.float()[:, None, None]
        if s["inv_freq"] is not None:
            y = _rotate32(y, cos, sin, c["inter"])
        return y.to(x.dtype)

    def store(pool, x):
        view = pool.transpose(2, 3) if c["layout"] else pool
        view[:, page, slot] = x

    store(s["k_pages"], ready(s["k"], s["k_gain"]))
    store(s["v_pages"], flat(s["v"]))
    out = {"k": s["k_pages"], "v": s["v_pages"]}
    if s["q"] is not None:
        flat(s["q_out"]).copy_(ready(s["q"], s["q_gain"]))
        out["q"] = s["q_out"]
    return out


def _copy_rows32(pool, layout, src, dst, rows):
    """Rows 0 .. rows[i] of page src[i] to page dst[i], in every layer."""
    ps = pool.shape[3] if layout else pool.shape[2]
    keep = torch.arange(ps, device=pool.device)[None] < rows[:, None]
    keep = keep[:, None, :, None] if layout else keep[:, :, None, None]
    pool[:, dst] = torch.where(keep[None], pool[:, src], pool[:, dst])


def _reorder32(s):
    c, table = s["case"], s["table"].long()
    ps, n_pages, (B, M) = c["page"], s["k_pages"].shape[1], s["table"].shape
    dev = table.device
    src = s["source"].long()
    keep = torch.where((src >= 0) & (src < B), s["keep"].long(), 0).clamp(0, M * ps)
    want = torch.maximum(s["want"].long().clamp(max=M * ps), keep)
    col, row = torch.arange(M, device=dev)[None], torch.arange(B, device=dev)
    full, kept, need = keep // ps, -(-keep // ps), -(-want // ps)
    mine = torch.where(col < kept[:, None], table[src.clamp(0, B - 1)], -1)
    good = (mine >= 0) & (mine < n_pages)
    whole = torch.zeros(n_pages + 1, device=dev, dtype=torch.bool)
    whole[torch.where(good & (col < full[:, None]), mine, n_pages)] = True
    part_col = (col == full[:, None]) & (col < kept[:, None]) & good
    part = torch.where(part_col, mine, n_pages)
    first = torch.full((n_pages + 1,), B, device=dev)
    first = first.scatter_reduce(0, part.flatten(), row[:, None].expand(B, M).flatten(), "amin")
    copied = part_col & (whole[part] | (first[part] != row[:, None]))
    held = (whole | (first < B))[:n_pages]
    free = torch.sort(held.int(), stable=True).indices            # the free pages first, in order
    n_free = n_pages - held.sum()
    grown = (col >= kept[:, None]) & (col < need[:, None])
    asked = copied | grown
    rank = asked.flatten().cumsum(0).view(B, M) - 1
    got = torch.where(rank < n_free, free[rank.clamp(0, n_pages - 1)], -1)
    new = torch.where(asked, got, torch.where(good, mine, -1))
    s["new_table"].copy_(new)
    s["missing"].copy_((asked.sum() - n_free).clamp(min=0))
    at = (copied & (new >= 0)).nonzero(as_tuple=True)
    for pool in (s["k_pages"], s["v_pages"]):
        _copy_rows32(pool, c["layout"], mine[at], new[at], (keep - full * ps)[at[0]])
    return {"k": s["k_pages"], "v": s["v_pages"], "table": s["new_table"], "missing": s["missing"]}


def _compact32(s):
    table, n_pages = s["table"].long(), s["k_pages"].shape[1]
    good = (table >= 0) & (table < n_pages)
    held = torch.zeros(n_pages + 1, device=table.device, dtype=torch.bool)
    held[torch.where(good, table, n_pages)] = True
    held = held[:n_pages]
    used = held.sum()
    page = torch.arange(n_pages, device=table.device)
    src = (held & (page >= used)).nonzero()[:, 0]
    dst = (~held & (page < used)).nonzero()[:, 0]
    to = page.clone()
    to[src] = dst
    s["new_table"].copy_(torch.where(good, to[table.clamp(0, n_pages - 1)], -1))
    s["used"].copy_(used)
    for pool in (s["k_pages"], s["v_pages"]):
        pool[:, dst] = pool[:, src]
    return {"k": s["k_pages"], "v": s["v_pages"], "table": s["new_table"], "used": s["used"]}


# what a pass cannot do without ----------------------------------------------------------------------------------------

def work(case):
    c = case
    hq, h, d, t = HEADS[c["heads"]]
    es, ps = 4 if t == "f32" else 2, c["page"]
    if c["op"] == "attend":
        lens, n = _lengths(c)
        seen = pairs = 0
        for kv, m in zip(lens, n):
            w = c["window"] or kv
            seen += min(kv, w + m - 1)
            # the positions that the new tokens see: kv - m + 1 .. kv each, at most w
            lo = kv - m + 1
            short = max(0, min(m, w - lo + 1))                     # tokens that see fewer than w or just w
            pairs += short * lo + short * (short - 1) // 2 + (m - short) * w
        return {"bytes": es * d * (2 * h * seen + 2 * hq * sum(n)) + 4 * sum(_pages(x, ps) for x in lens),
                "flops": 4 * hq * d * pairs}
    if c["op"] == "append":
        n, L = sum(_lengths(c)[1]), c["L"]
        moved = 2 * es * d * L * n * (2 * h + (0 if c["plain"] else hq))
        return {"bytes": moved, "flops": 0 if c["plain"] else 8 * d * L * n * (h + hq)}
    row = 2 * es * d * h * c["L"]                                  # keys and values of a position
    if c["op"] == "reorder":
        old, src, keep, want = _parents(c)
        whole, first, copied = set(), {}, 0
        for b, s in enumerate(src):
            whole |= {(s, j) for j in range(keep[b] // ps)}
            if keep[b] % ps:
                first.setdefault((s, keep[b] // ps), b)
        for b, s in enumerate(src):
            at = (s, keep[b] // ps)
            if keep[b] % ps and (at in whole or first[at] != b):
                copied += keep[b] % ps
        return {"bytes": 2 * row * copied + 8 * sum(_pages(x, ps) for x in old) + 16 * c["B"], "flops": 0}
    lens, alive = _alive(c)
    total, used = sum(_pages(x, ps) for x in lens) + 3, sum(_pages(x, ps) for x in alive)
    # pages in use lie anywhere: of the places past the first `used`, that share of them holds one
    return {"bytes": 2 * row * ps * used * (total - used) / total + 8 * used, "flops": 0}


# 64-bit results -------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "reorder": _exact_reorder,
            "compact": _exact_compact}[case["op"]](case, s)


def _spans(c):
    lens, n = _lengths(c)
    at = 0
    for b, (kv, m) in enumerate(zip(lens, n)):
        yield b, at, kv, m
        at += m


def _exact_attend(c, s):
    hq, h, d, _ = HEADS[c["heads"]]
    G, ps = hq // h, c["page"]
    q = s["q"].reshape(-1, hq, d)
    o = torch.zeros(q.shape, device="cuda", dtype=torch.float64)
    for b, at, kv, m in _spans(c):
        ids = s["table"][b, :_pages(kv, ps)].long()
        for x in range(h):
            pick = (lambda p: (p[ids, x] if c["layout"] else p[ids, :, x]).reshape(-1, d)[:kv].double())
            key, val = pick(s["k_pages"]), pick(s["v_pages"])
            far = torch.arange(kv - m, kv, device="cuda")[:, None] - torch.arange(kv, device="cuda")[None]
            hide = far < 0
            if c["window"]:
                hide |= far >= c["window"]
            for y in range(x * G, (x + 1) * G):
                sc = (q[at:at + m, y].double() @ key.T) / math.sqrt(d)
                o[at:at + m, y] = torch.softmax(sc.masked_fill_(hide, -math.inf), -1) @ val
    return {"o": o.view(s["o"].shape)}


def _exact_append(c, s):
    ps, (hq, h, d, _) = c["page"], HEADS[c["heads"]]
    out = {x: s[x + "_pages"].double() for x in ("k", "v")}
    if s["q"] is not None:
        out["q"] = torch.zeros(s["q_out"].shape, device="cuda", dtype=torch.float64)
    half = d // 2
    for l in range(c["L"]):
        for b, at, kv, m in _spans(c):
            pos = torch.arange(kv - m, kv, device="cuda")
            for name, x in (("k", s["k"]), ("v", s["v"]), ("q", s["q"])):
                if x is None:
                    continue
                y = (x[l, at:at + m] if c["ragged"] else x[l, b]).double()
                gain = s.get(name + "_gain")
                if gain is not None:
                    y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * gain[l].double()
                if s["inv_freq"] is not None and name != "v":
                    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64),
                                       pos.double()[:, None, None] * s["inv_freq"].double())
                    if c["inter"]:
                        y = torch.view_as_real(torch.view_as_complex(y.reshape(m, -1, half, 2)) * turn).reshape(y.shape)
                    else:
                        z = torch.complex(y[..., :half], y[..., half:]) * turn
                        y = torch.cat((z.real, z.imag), -1)
                if name == "q":
                    if c["ragged"]:
                        out["q"][l, at:at + m] = y
                    else:
                        out["q"][l, b] = y
                else:
                    pool = out[name][l].transpose(1, 2) if c["layout"] else out[name][l]
                    pool[s["table"][b].long()[pos // ps], pos % ps] = y
    return out


def _exact_reorder(c, s):
    ps, n_pages = c["page"], s["k_pages"].shape[1]
    _, src, keep, want = _parents(c)
    table = s["table"].tolist()
    rows, whole, first = [], set(), {}
    for b, x in enumerate(src):
        n = _pages(keep[b], ps)
        rows.append(table[x][:n] if x >= 0 else [])
        whole.update(rows[b][:keep[b] // ps])
        if keep[b] % ps:
            first.setdefault(rows[b][-1], b)
    free = iter([p for p in range(n_pages) if p not in whole and p not in first])
    pools = {x: s[x + "_pages"].double() for x in ("k", "v")}
    missing, pairs = 0, []
    for b in range(len(src)):
        new = list(rows[b])
        if keep[b] % ps and (new[-1] in whole or first[new[-1]] != b):
            p = next(free, -1)
            if p >= 0:
                pairs.append((new[-1], p, keep[b] % ps))
            missing += p < 0
            new[-1] = p
        while len(new) < _pages(want[b], ps):
            p = next(free, -1)
            missing += p < 0
            new.append(p)
        table[b] = new + [-1] * (len(table[b]) - len(new))
    for x, y, r in pairs:
        for pool in pools.values():
            if c["layout"]:
                pool[:, y, :, :r] = pool[:, x, :, :r]
            else:
                pool[:, y, :r] = pool[:, x, :r]
    return {**pools, "table": _ints(table), "missing": _ints([missing])}


def _exact_compact(c, s):
    table = s["table"].tolist()
    held = sorted({p for row in table for p in row if p >= 0})
    used = len(held)
    there = set(held)
    to = dict(zip([p for p in held if p >= used], [p for p in range(used) if p not in there]))
    pools = {x: s[x + "_pages"].double() for x in ("k", "v")}
    for x, y in to.items():
        for pool in pools.values():
            pool[:, y] = pool[:, x]
    return {**pools, "table": _ints([[to.get(p, p) for p in row] for row in table]), "used": _ints([used])}
