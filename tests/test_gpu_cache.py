"""The paged cache on the GPU against its float64 oracle: attention of new
tokens over pages, normed and rotated appends, reordering, compaction, and a
run of them together.

Bounds.  A rounding to t is off by at most eps(t) / 2 of the value.  Attention:
scores are sums of D fp32 products and one fused multiply-add, so their error
(and the weights' relative error, twice for weight and sum) is at most
(D + 4) 2^-24 S for S the largest sum of scaled |q k|; the sums over N
positions add (N + 8) 2^-24; all of it times A = sum of softmax |v|.  bf16 adds
the rounding of the probabilities, 2^-8 A, and the result's, 2^-8 of it; where a
row's sum takes the rounded probabilities too (tiles of 128 rows) it is off by at
most 2^-8 of itself, and so the quotient by another 2^-8 of the result (and these
errors of each other, under 2^-15 A).
Append: the fp32 steps (a sum of squares over D in lanes of 16, square root,
quotient, two products, the turn's three roundings and an angle within 2^-25
turns) stay under 2^-19 of |a| + |b| of the pair.
"""
import numpy as np
import pytest

from oracle import cache as ref
from paper_2607_28979_amd import binding as mb

pytestmark = pytest.mark.gpu

KEEP = -3.75      # what unwritten rows hold
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _dt(t):
    import torch
    return torch.bfloat16 if t == "bf16" else torch.float32


def _rand(rng, shape, t, scale=1.0):
    """(device tensor, its float64 values)."""
    import torch
    x = torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).cuda().to(_dt(t))
    return x, x.double().cpu().numpy()


def _i32(v):
    import torch
    return torch.tensor(np.ascontiguousarray(v), dtype=torch.int32, device="cuda")


def _np(x):
    return x.double().cpu().numpy()


class Cache:
    """Pools with every position drawn, pages of the sequences at random places;
    positions past kv_len are NaN."""

    def __init__(self, rng, kv, ps, H, D, t, layout=0, L=None, spare=3, stale=True, max_pages=None, filled=True):
        import torch
        self.kv, self.ps, self.layout = list(kv), ps, layout
        counts = [-(-max(n, 0) // ps) for n in kv]
        self.n_pages = sum(counts) + spare
        order, at = rng.permutation(self.n_pages), 0
        self.table = np.full((len(kv), max_pages or max(1, max(counts) + 1)), -1, np.int32)
        for b, n in enumerate(counts):
            self.table[b, :n] = order[at:at + n]
            at += n
        page = (H, ps, D) if layout else (ps, H, D)
        lead = () if L is None else (L,)
        self.k, _ = _rand(rng, lead + (self.n_pages,) + page, t)
        self.v, _ = _rand(rng, lead + (self.n_pages,) + page, t)
        if stale:      # what a recycled page may hold
            held = torch.zeros(self.n_pages, ps, dtype=torch.bool, device="cuda")
            for b, n in enumerate(kv):
                for j in range(n):
                    held[self.table[b, j // ps], j % ps] = True
            m = (held[:, None, :, None] if layout else held[:, :, None, None])
            for pool in (self.k, self.v):
                pool.masked_fill_(~m, float("nan"))
        self.d_table, self.d_kv = _i32(self.table), _i32(self.kv)

    def host(self):
        return _np(self.k), _np(self.v)


def _bound(t, want, mag, smax, D, n, rounded_sum=False):
    b = HALF[t] * np.abs(want) + mag * (2 * (D + 4) * smax + 2 * (n + 8)) * 2.0 ** -24
    b = b + (HALF["bf16"] * mag if t == "bf16" else 0) + 1e-30
    return b + (HALF["bf16"] * np.abs(want) + 2.0 ** -15 * mag if rounded_sum else 0)


def _attend(c, q, counts=None, window=0, scale=None, max_new=None, o=None, **kw):
    """(device o, checked against the oracle).  counts: packed new tokens."""
    import torch
    t = "bf16" if q.dtype == torch.bfloat16 else "f32"
    o = torch.full_like(q, KEEP) if o is None else o
    start = None if counts is None else np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    mb.paged_attention(q, c.k, c.v, c.d_table, c.d_kv, o, new_start=None if start is None else _i32(start),
                       max_new=max_new, window=window, scale=scale, page_layout=c.layout, **kw)
    torch.cuda.synchronize()
    H, D = q.shape[-2:]
    k, v = c.host()
    flat = np.full((int(np.prod(q.shape[:-2])), H, D), KEEP)
    mx = (q.shape[1] if start is None else q.shape[0]) if max_new is None else max_new
    want, mag, smax = ref.paged_attention(_np(q).reshape(flat.shape), k, v, c.table, c.kv, flat, start, mx, window, scale, c.layout)
    got = _np(o).reshape(flat.shape)
    G, B = H // c.k.shape[-3 if c.layout else -2], len(c.kv)
    wide = mx * G > 32 and flat.shape[0] * G > 32 * B      # tiles of 128 rows
    bound = _bound(t, want, mag, smax, D, max(c.kv), t == "bf16" and wide)
    bad = ~(np.abs(got - want) <= bound) & ~(np.isnan(got) & np.isnan(want))
    worst = np.unravel_index(np.argmax(bad), bad.shape)
    assert not bad.any(), (int(bad.sum()), worst, got[worst], want[worst], bound[worst])
    return o


ATTEND = [  # kv lengths, new tokens (int: each, list: packed), H_q, H_kv, D, page, layout, window, type
    ([1, 2, 17, 64, 65, 200], 1, 28, 4, 128, 16, 0, 0, "bf16"),
    ([0, 1, 31, 32, 33, 127, 300], 1, 12, 2, 128, 32, 1, 0, "bf16"),
    ([700, 3], 1, 14, 2, 64, 64, 0, 0, "bf16"),
    ([129, 64], 1, 4, 4, 64, 16, 1, 0, "bf16"),
    ([90, 40], 1, 48, 1, 128, 16, 0, 0, "bf16"),              # more query heads than a tile of 32 rows
    ([70, 5, 33], 5, 14, 2, 64, 16, 0, 0, "bf16"),
    ([150, 40], 37, 12, 2, 128, 32, 0, 0, "bf16"),
    ([130, 1, 0, 250], [100, 1, 0, 7], 28, 4, 128, 64, 0, 0, "bf16"),
    ([260], 260, 4, 2, 128, 128, 1, 0, "bf16"),
    ([20, 3], 30, 4, 2, 64, 16, 0, 0, "bf16"),                # more new tokens than positions: empty rows
    ([400, 90], 1, 14, 2, 64, 16, 0, 50, "bf16"),
    ([300, 64], [90, 3], 12, 2, 128, 16, 0, 33, "bf16"),
    ([200], 128, 4, 4, 64, 1024, 0, 1, "bf16"),
    ([1, 17, 333], 1, 12, 12, 64, 16, 0, 0, "f32"),
    ([100, 64, 0], [64, 5, 0], 12, 12, 64, 16, 1, 0, "f32"),
    ([140, 9], 20, 12, 2, 128, 32, 0, 0, "f32"),
    ([180], 70, 4, 2, 128, 16, 0, 21, "f32"),
]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "kv%s-new%s-%d/%d-D%d-p%d-l%d-w%d-%s" % (
    "_".join(map(str, c[0])), str(c[1]).replace(", ", "_"), *c[2:]))
@pytest.mark.parametrize("cut", [False, True])
def test_attention(case, cut):
    kv, new, Hq, H, D, ps, layout, window, t = case
    print("case attention", case, "cut", cut, flush=True)
    rng = np.random.default_rng(len(kv) * 1000 + kv[0])
    # rows far longer than any sequence make the call cut them where it may
    c = Cache(rng, kv, ps, H, D, t, layout, max_pages=max(1, 4096 // ps) if cut else None)
    packed = isinstance(new, list)
    q, _ = _rand(rng, (sum(new) + 2 if packed else len(kv),) + (() if packed else (new,)) + (Hq, D), t)
    o = _attend(c, q, new if packed else None, window, scratch=None if cut else False)
    if packed:
        assert (o[sum(new):] == KEEP).all()     # rows behind the last sequence


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_attention_every_length(t):
    """Single tokens on every length from 0 to 140, and every count of new tokens
    on one length."""
    rng = np.random.default_rng(7)
    kv = list(range(141))
    c = Cache(rng, kv, 16, 2, 64, t)
    q, _ = _rand(rng, (len(kv), 1, 6, 64), t)
    _attend(c, q)
    counts = list(range(0, 40))
    c = Cache(rng, [45] * len(counts), 32, 2, 64, t, 1)
    q, _ = _rand(rng, (sum(counts), 4, 64), t)
    _attend(c, q, counts)
    _attend(c, q, counts, max_new=max(counts))


def test_attention_holes_and_bad_entries():
    """Entries outside the pool are holes: inside a sequence, at its end, all of
    it; keys and values of other pages are NaN."""
    for t, n in (("bf16", 1), ("bf16", 50), ("f32", 20)):
        rng = np.random.default_rng(3)
        c = Cache(rng, [200, 130, 60, 300], 16, 2, 128, t)
        c.table[0, [2, 3, 7]] = [-1, c.n_pages, 1 << 30]
        c.table[1, 8] = -5
        c.table[2, :] = -1
        c.table[3, 4:9] = -(1 << 31)
        c.d_table = _i32(c.table)
        q, _ = _rand(rng, (4, n, 4, 128), t)
        print("case holes", t, n, flush=True)
        _attend(c, q)
        _attend(c, q, window=70)


@pytest.mark.parametrize("t,new", [("bf16", 40), ("bf16", 3), ("f32", 40)])
def test_attention_values_that_are_not_finite(t, new):
    """A NaN or infinite value (or key) reaches the tokens that see it and no
    others: here at positions that only the later new tokens see."""
    import torch
    rng = np.random.default_rng(5)
    c = Cache(rng, [100, 64], 16, 2, 64, t)
    for b, pos, pool, x in ((0, 100 - new + 2, "v", float("inf")), (1, 63, "v", float("nan")), (1, 64 - new + 1, "k", float("nan"))):
        getattr(c, pool)[c.table[b, pos // 16], pos % 16, 1] = x
    q, _ = _rand(rng, (2, new, 4, 64), t)
    o = torch.full_like(q, KEEP)
    mb.paged_attention(q, c.k, c.v, c.d_table, c.d_kv, o)
    got = _np(o)
    assert np.isfinite(got[0, :2]).all() and np.isfinite(got[1, :1]).all()
    assert not np.isfinite(got[0, 2:, 2:]).any() and np.isnan(got[1, 1:, 2:]).all()
    assert np.isfinite(got[:, :, :2]).all()           # the other KV head's queries
    k, v = c.host()
    clean_k, clean_v = np.nan_to_num(k, posinf=0), np.nan_to_num(v, posinf=0)
    flat = _np(q).reshape(-1, 4, 64)
    want, mag, smax = ref.paged_attention(flat, clean_k, clean_v, c.table, c.kv, flat, max_new=new)
    fine = np.isfinite(got.reshape(flat.shape))
    assert (np.abs(got.reshape(flat.shape) - want) <= _bound(t, want, mag, smax, 64, 100, t == "bf16" and new > 16))[fine].all()


def test_attention_strides_and_layouts():
    """Queries as a slice of a fused projection, outputs in head-major memory and
    with a gap between tokens; the same bits as from contiguous rows."""
    import torch
    for t in ("bf16", "f32"):
        for n in (1, 33):
            rng = np.random.default_rng(n)
            c = Cache(rng, [80, 41, 5], 16, 2, 64, t)
            fused, _ = _rand(rng, (3, n, 8 + 2 * 2, 64), t)
            q = fused[:, :, :8]
            a = _attend(c, q.contiguous())
            head_major = torch.full((3, 8, n, 64), KEEP, dtype=_dt(t), device="cuda")
            assert torch.equal(_attend(c, q, o=head_major.transpose(1, 2)), a)
            wide = torch.full((3, n, 9, 64), KEEP, dtype=_dt(t), device="cuda")
            assert torch.equal(_attend(c, q, o=wide[:, :, :8]), a) and (wide[:, :, 8] == KEEP).all()


def test_attention_scale_and_large_scores():
    rng = np.random.default_rng(11)
    for t, n in (("bf16", 1), ("bf16", 40), ("f32", 9)):
        c = Cache(rng, [150, 64], 16, 2, 64, t)
        q, _ = _rand(rng, (2, n, 4, 64), t)
        _attend(c, q, scale=1.0)
        _attend(c, q, scale=0.01)
        _attend(c, q * 64, scale=0.5)


def test_attention_long_cut_equals_uncut():
    """A long context cut over workgroups, and whole: the same within the order of
    fp32 sums, and each the same bits every time."""
    import torch
    for t, Hq, H, D, n in (("bf16", 28, 4, 128, 1), ("bf16", 12, 2, 128, 37), ("f32", 12, 2, 128, 3)):
        g = torch.Generator(device="cuda").manual_seed(1)
        kv, ps = 30011, 64
        pages = -(-kv // ps)
        pool = [torch.randn((pages, ps, H, D), generator=g, device="cuda").to(_dt(t)) for _ in range(2)]
        table = torch.randperm(pages, generator=g, device="cuda").int()[None]
        q = torch.randn((1, n, Hq, D), generator=g, device="cuda").to(_dt(t))
        outs = []
        for scratch in (None, False, None, False):
            o = torch.full_like(q, KEEP)
            mb.paged_attention(q, *pool, table, _i32([kv]), o, scratch=scratch)
            outs.append(o)
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
        k, v = (x[table[0].long()].reshape(-1, H, D)[:kv].double() for x in pool)
        G = Hq // H
        for o in outs[:2]:
            for h in range(Hq):
                s = (q[0, :, h].double() @ k[:, h // G].T) / D ** 0.5
                u = torch.arange(kv - n, kv, device="cuda")
                s.masked_fill_(torch.arange(kv, device="cuda")[None] > u[:, None], -float("inf"))
                p = torch.softmax(s, -1)
                want, mag = p @ v[:, h // G], p @ v[:, h // G].abs()
                smax = (q[0, :, h].double().abs() @ k[:, h // G].abs().T).amax() / D ** 0.5
                bound = _bound(t, want.cpu().numpy(), mag.cpu().numpy(), float(smax), D, kv, t == "bf16" and n * G > 32)
                assert (np.abs((o[0, :, h].double() - want).cpu().numpy()) <= bound).all(), (t, h)


@pytest.mark.parametrize("B,t,new", [(70, "bf16", 1), (70, "f32", 2), (90, "bf16", 20), (512, "bf16", 1), (513, "bf16", 1), (600, "f32", 1),
                                     (1100, "bf16", 1), (1030, "bf16", 17), (1030, "f32", 3)])
def test_attention_of_many_sequences(B, t, new):
    """More sequences than a wave has lanes (their lengths are shared out by several per
    lane), and more than are shared out at a time; a few long ones among empty ones."""
    rng = np.random.default_rng(B)
    kv = rng.integers(0, 40, B)
    kv[rng.integers(0, B, 12)] = 0
    kv[[0, B // 2, B - 1]] = [900, 0, 1300]
    kv[63:66] = [500, 0, 333]
    c = Cache(rng, kv.tolist(), 16, 1, 64, t, stale=False, max_pages=256)
    print("case many", B, t, new, flush=True)
    q, _ = _rand(rng, (B, new, 2, 64), t)
    _attend(c, q)
    counts = rng.integers(0, new + 1, B)
    q, _ = _rand(rng, (int(counts.sum()) + 1, 2, 64), t)
    o = _attend(c, q, counts.tolist(), max_new=new)
    assert (o[int(counts.sum()):] == KEEP).all()


@pytest.mark.parametrize("t,n", [("bf16", 1), ("bf16", 60), ("f32", 9)])
def test_attention_of_starts_that_do_not_ascend(t, n):
    """Starts out of order name rows twice, more than the call has: the rows of no sequence
    and the pools stay as they are, and the next call is right."""
    import torch
    rng = np.random.default_rng(n)
    c = Cache(rng, [1500] * 40, 16, 2, 128, t, stale=False, max_pages=128)
    q, _ = _rand(rng, (n + 2, 12, 128), t)
    k, v = c.k.clone(), c.v.clone()
    o = torch.full_like(q, KEEP)
    start = [0, n] * 20 + [0]
    print("case starts", t, n, flush=True)
    mb.paged_attention(q, c.k, c.v, c.d_table, c.d_kv, o, new_start=_i32(start))
    mb.paged_attention(q, c.k, c.v, c.d_table, c.d_kv, o, new_start=_i32([s - 5 for s in start[::-1]]))
    torch.cuda.synchronize()
    assert (o[n:] == KEEP).all() and torch.equal(k, c.k) and torch.equal(v, c.v)
    _attend(c, q[:n], [0] * 39 + [n])


@pytest.mark.parametrize("t,B,most", [("bf16", 40, 1), ("bf16", 100, 30), ("bf16", 40, 250), ("f32", 40, 1), ("f32", 90, 60), ("bf16", 600, 12),
                                      ("bf16", 530, 900), ("f32", 1040, 40)])
@pytest.mark.parametrize("cut", [False, True])
def test_attention_of_packed_tokens_without_a_bound(t, B, most, cut):
    """Packed tokens and no max_new: nearly all of the tiles that it admits are none, and one
    sequence has most of the tokens."""
    rng = np.random.default_rng(B + most)
    counts = rng.integers(0, 3, B)
    counts[[0, B - 1]] = 1
    counts[B // 3] = most
    kv = counts + rng.integers(0, 60, B)
    kv[[1, B // 2]] = [1200, 700]
    c = Cache(rng, kv.tolist(), 16, 2, 64, t, stale=False, max_pages=128 if cut else None)
    print("case loose", t, B, most, cut, flush=True)
    q, _ = _rand(rng, (int(counts.sum()) + 1, 12, 64), t)
    loose = _attend(c, q, counts.tolist(), scratch=None if cut else False)
    assert (loose[int(counts.sum()):] == KEEP).all()
    _attend(c, q, counts.tolist(), max_new=most, scratch=None if cut else False, window=37)


def test_attention_repeats_itself_over_two_streams():
    """Calls on two streams at once, each with its own partial sums, give the bits of calls
    one after the other."""
    import torch
    rng = np.random.default_rng(17)
    c = [Cache(rng, [1500, 40, 2900], 16, 2, 128, "bf16", max_pages=200) for _ in range(2)]
    for n in (1, 30):
        q = [_rand(rng, (3, n, 12, 128), "bf16")[0] for _ in range(2)]
        alone = [_attend(c[i], q[i]) for i in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        outs = [[torch.full_like(x, KEEP) for _ in range(6)] for x in q]
        torch.cuda.synchronize()
        for j in range(6):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    mb.paged_attention(q[i], c[i].k, c[i].v, c[i].d_table, c[i].d_kv, outs[i][j])
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(x, alone[i]) for x in outs[i]), (n, i)


def test_two_graphs_at_once():
    """Two captured calls, replayed on two streams at once, share no partial sums."""
    import torch
    rng = np.random.default_rng(19)
    c = Cache(rng, [1500, 40, 2900], 16, 2, 128, "bf16", max_pages=200)
    q = [_rand(rng, (3, 1, 12, 128), "bf16")[0] for _ in range(2)]
    alone = [_attend(c, x) for x in q]
    outs, graphs = [torch.full_like(x, KEEP) for x in q], []
    for x, o in zip(q, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mb.paged_attention(x, c.k, c.v, c.d_table, c.d_kv, o)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for o in outs:
            o.fill_(KEEP)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, a) for o, a in zip(outs, alone))


def test_offsets_past_32_bits():
    """Pages past 2^31 elements of a pool, written and attended."""
    import torch
    n_pages, ps, H, D = 70001, 64, 4, 128
    k = torch.empty((n_pages, ps, H, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    table = _i32([[70000, 3], [69999, 65537]])
    rng = np.random.default_rng(2)
    x, _ = _rand(rng, (2, 100, H, D), "bf16")
    y, _ = _rand(rng, (2, 100, H, D), "bf16")
    kv = _i32([100, 100])
    mb.cache_append(None, x, y, None, k, v, table, kv)
    small = Cache(rng, [100, 100], ps, H, D, "bf16", stale=False)
    for b in range(2):
        for j in range(2):
            small.k[int(small.table[b, j])] = k[int(table[b, j])]
            small.v[int(small.table[b, j])] = v[int(table[b, j])]
    for n in (1, 60):
        q, _ = _rand(rng, (2, n, 28, D), "bf16")
        o = torch.full_like(q, KEEP)
        mb.paged_attention(q, k, v, table, kv, o)
        assert torch.equal(o, _attend(small, q))
    new, used = torch.empty_like(table), _i32([0])
    before = [k[int(table[b, 0])].clone() for b in range(2)]
    mb.cache_compact(k, v, table, new, used)
    assert new.tolist() == [[2, 3], [1, 0]] and int(used) == 4
    assert torch.equal(k[2], before[0]) and torch.equal(k[1], before[1])


APPEND = [  # kv, new, H_q (0: none), H_kv, D, page, layout, L, norm, rotary dims (0: none), interleaved, type, rows
    ([5, 1, 40], 1, 28, 4, 128, 16, 0, None, True, 128, False, "bf16", "bthd"),
    ([33, 64], 33, 12, 2, 128, 32, 1, None, False, 128, False, "bf16", "bhtd"),
    ([20, 4, 0, 17], [20, 3, 0, 1], 14, 2, 64, 16, 0, None, True, 64, True, "bf16", "bthd"),
    ([50], 50, 0, 4, 128, 16, 0, 5, False, 0, False, "bf16", "bhtd"),
    ([9, 30], 9, 3, 1, 80, 16, 0, 2, True, 32, False, "bf16", "bthd"),
    ([9, 30], 9, 3, 3, 256, 16, 1, 2, True, 64, True, "bf16", "bthd"),
    ([7, 25], 7, 2, 1, 16, 16, 0, None, True, 16, False, "bf16", "bthd"),
    ([5, 2], 8, 4, 4, 32, 16, 0, None, False, 32, False, "bf16", "bthd"),      # negative positions: not stored
    ([40, 1], 1, 12, 12, 64, 16, 0, None, False, 64, False, "f32", "bthd"),
    ([70], 70, 12, 2, 128, 32, 1, 3, True, 96, True, "f32", "bhtd"),
    ([700, 690], 690, 2, 1, 64, 64, 0, 2, True, 64, False, "bf16", "bthd"),     # several tokens per workgroup
]


def _append_case(case, seed=0, positions=None, kv_add=0):
    import torch
    kv, new, Hq, H, D, ps, layout, L, norm, rot, inter, t, rows = case
    rng = np.random.default_rng(seed + sum(kv))
    c = Cache(rng, [n + kv_add for n in kv], ps, H, D, t, layout, L, stale=False)
    packed = isinstance(new, list)
    lead = () if L is None else (L,)

    def make(h):
        if packed:
            return _rand(rng, lead + (sum(new), h, D), t)[0]
        if rows == "bhtd":
            return _rand(rng, lead + (len(kv), h, new, D), t)[0].transpose(-3, -2)
        return _rand(rng, lead + (len(kv), new, h, D), t)[0]

    q = make(Hq) if Hq else None
    k, v = make(H), make(H)
    gains = [_rand(rng, lead + (D,), t)[0] if norm else None for _ in range(2)]
    f = torch.from_numpy((10000.0 ** -(np.arange(rot // 2) / max(1, rot // 2))).astype(np.float32)).cuda() if rot else None
    q_out = torch.full(q.shape, KEEP, dtype=q.dtype, device="cuda") if Hq else None
    start = np.concatenate([[0], np.cumsum(new)]) if packed else None
    return c, q, k, v, q_out, gains, f, start


def _check_append(case, c, q, k, v, q_out, gains, f, start, before, positions=None):
    kv, new, Hq, H, D, ps, layout, L, norm, rot, inter, t, rows = case
    n_rows = k[0].numel() // (H * D) if L is not None else k.numel() // (H * D)
    lay = lambda x, h: None if x is None else _np(x).reshape((L or 1, n_rows, h, D))     # noqa: E731
    pool = lambda x: x if L is not None else x[None]                                      # noqa: E731
    g = [None if x is None else _np(x).reshape(L or 1, D) for x in gains]
    want = ref.cache_append(lay(q, Hq), lay(k, H), lay(v, H), None if q is None else np.full((L or 1, n_rows, Hq, D), KEEP),
                            pool(before[0]), pool(before[1]), c.table, c.kv, start,
                            (new if not isinstance(new, list) else n_rows), g[0], g[1], 1e-6,
                            None if f is None else _np(f), inter, positions, layout)
    got = (lay(q_out, Hq), pool(_np(c.k)), pool(_np(c.v)))
    for name, x, y in zip(("q", "k", "v"), got, want):
        if y is None:
            continue
        if name == "v" or (f is None and not norm):
            assert np.array_equal(x, y), name
            continue
        r = rot or D
        mag = np.abs(y).copy()          # |a| + |b| of each pair, at most sqrt 2 of the turned pair's
        a = np.abs(y[..., :r])
        pair = (a[..., 0::2] + a[..., 1::2]) if inter else (a[..., :r // 2] + a[..., r // 2:])
        mag[..., :r] = 1.5 * (np.repeat(pair, 2, -1) if inter else np.concatenate([pair, pair], -1))
        bound = HALF[t] * np.abs(y) * 1.01 + 2.0 ** -19 * mag
        same = np.zeros(y.shape, bool) if name == "q" else y == pool(before[0])
        bad = ~(np.abs(x - y) <= bound) & ~(same & (x == y))
        assert not bad.any(), (name, int(bad.sum()), np.unravel_index(np.argmax(bad), bad.shape))


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(x).replace(", ", "_") for x in c))
def test_append(case):
    import torch
    print("case append", case, flush=True)
    a = _append_case(case)
    c, q, k, v, q_out, gains, f, start = a
    before = c.host()
    mb.cache_append(q, k, v, q_out, c.k, c.v, c.d_table, c.d_kv, new_start=None if start is None else _i32(start),
                    q_gain=gains[0], k_gain=gains[1], inv_freq=f, interleaved=case[10], page_layout=case[6])
    torch.cuda.synchronize()
    _check_append(case, *a, before)


@pytest.mark.parametrize("t,L,D,n,ps", [("bf16", 1, 128, 8192, 64), ("f32", 1, 64, 8200, 16), ("bf16", 3, 32, 13000, 16)])
def test_append_of_many_equals_parts(t, L, D, n, ps):
    """A call that writes more than the caches hold, and the same tokens in parts: the same
    bits, in both of which every row is written once."""
    import torch
    Hq, H = 28, 4
    g = torch.Generator(device="cuda").manual_seed(n)
    lead = () if L == 1 else (L,)
    x = torch.randn(lead + (1, n, Hq + 2 * H, D), generator=g, device="cuda").to(_dt(t))
    f = torch.rand(D // 2, generator=g, device="cuda")
    gain = (1 + 0.1 * torch.randn((L, D), generator=g, device="cuda")).to(_dt(t))
    pages = -(-n // ps)
    table = torch.randperm(pages + 2, generator=g, device="cuda").int()[:pages][None].contiguous()
    assert n * L * (Hq + 2 * H) * D * x.element_size() > 64 << 20
    out = []
    for part in (n, 1025):
        k, v = (torch.full(lead + (pages + 2, ps, H, D), KEEP, device="cuda", dtype=_dt(t)) for _ in range(2))
        qo = torch.full(lead + (1, n, Hq, D), KEEP, device="cuda", dtype=_dt(t))
        for at in range(0, n, part):
            m = slice(at, min(at + part, n))
            y = x[..., m, :, :]
            mb.cache_append(y[..., :Hq, :], y[..., Hq:Hq + H, :], y[..., Hq + H:, :], qo[..., m, :, :], k, v, table, _i32([m.stop]),
                            inv_freq=f, q_gain=gain, k_gain=gain)
        out.append((k, v, qo))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert int((out[0][1] == KEEP).all(-1).all(-1).sum()) == L * ((pages + 2) * ps - n)


@pytest.mark.parametrize("B,most,L,t", [(3, 40, 1, "bf16"), (64, 9, 2, "bf16"), (65, 300, 1, "f32"), (700, 5, 1, "bf16"), (5000, 700, 1, "bf16")])
def test_append_of_packed_tokens_without_a_bound(B, most, L, t):
    """Packed tokens and no max_new, whose sequences are found row by row, give the bits of
    the call with the bound: sequences of none, rows before the first and behind the last,
    holes, given positions."""
    import torch
    rng = np.random.default_rng(B)
    counts = rng.integers(0, 2, B)
    counts[[0, B - 1]] = 1, 0
    counts[2 * B // 3] = most
    start = 2 + np.concatenate([[0], np.cumsum(counts)])
    kv = counts + rng.integers(-1, 30, B)
    c = Cache(rng, np.maximum(kv, 0).tolist(), 16, 2, 32, t, L=L, stale=False)
    c.table[rng.integers(0, B, 2), 0] = [-1, c.n_pages]
    table, kv = _i32(c.table), _i32(kv)
    n = int(start[-1]) + 3
    q, k, v = (_rand(rng, (L, n, h, 32), t)[0] for h in (6, 2, 2))
    f, pos = torch.rand(8, device="cuda"), _i32(rng.integers(0, 1000, n))
    out = []
    for bound in (most, None):
        for given in (None, pos):
            pools, qo = (c.k.clone(), c.v.clone()), torch.full_like(q, KEEP)
            mb.cache_append(q, k, v, qo, *pools, table, kv, new_start=_i32(start), max_new=bound, inv_freq=f, positions=given)
            assert (qo[:, :2] == KEEP).all() and (qo[:, n - 3:] == KEEP).all()
            out.append((qo, *pools))
    assert all(torch.equal(a, b) for x, y in ((0, 2), (1, 3)) for a, b in zip(out[x], out[y]))
    assert not torch.equal(out[0][0], out[1][0]) and not torch.equal(out[0][1], c.k)
    # starts out of order: rows and places of some sequence or none, nothing else
    qo = torch.full_like(q, KEEP)
    mb.cache_append(q, k, v, qo, c.k, c.v, table, kv, new_start=_i32(rng.permutation(start) - 4), inv_freq=f)
    torch.cuda.synchronize()
    assert torch.isfinite(qo).all() and torch.isfinite(c.k).all() and torch.isfinite(c.v).all()


def test_append_far_positions_and_given_ones():
    """Angles of positions near 2^20 from the places, and of given positions (the
    places then at the sequence's end, as ever)."""
    import torch
    case = ([30, 12], 5, 2, 1, 64, 16, 0, None, False, 64, False, "f32", "bthd")
    a = _append_case(case)
    c, q, k, v, q_out, gains, f, start = a
    pos = np.array([0, 1, 999983, 1048575, 31, 2 ** 30, 2 ** 31 - 1, 7, 65536, 123456789], np.int32)
    before = c.host()
    mb.cache_append(q, k, v, q_out, c.k, c.v, c.d_table, c.d_kv, inv_freq=f, positions=_i32(pos))
    torch.cuda.synchronize()
    _check_append(case, *a, before, positions=pos)


def test_append_in_place_queries_of_a_fused_tensor():
    import torch
    rng = np.random.default_rng(4)
    for t in ("bf16", "f32"):
        c = Cache(rng, [20, 9], 16, 2, 64, t, stale=False)
        fused, _ = _rand(rng, (2, 9, 8 + 4, 64), t)
        keep = fused.clone()
        f = torch.from_numpy((0.5 ** np.arange(32)).astype(np.float32)).cuda()
        q, k, v = fused[:, :, :8], fused[:, :, 8:10], fused[:, :, 10:]
        other = torch.zeros((2, 9, 8, 64), dtype=_dt(t), device="cuda")
        kp, vp = c.k.clone(), c.v.clone()
        mb.cache_append(q, k, v, other, kp, vp, c.d_table, c.d_kv, inv_freq=f)
        mb.cache_append(q, k, v, q, c.k, c.v, c.d_table, c.d_kv, inv_freq=f)
        assert torch.equal(fused[:, :, :8], other) and torch.equal(fused[:, :, 8:], keep[:, :, 8:])
        assert torch.equal(kp, c.k) and torch.equal(vp, c.v)


def test_append_holes():
    """Tokens whose page is a hole are not stored, their queries are written."""
    import torch
    case = ([40, 33], 20, 4, 2, 64, 16, 0, None, True, 64, False, "bf16", "bthd")
    a = _append_case(case)
    c, q, k, v, q_out, gains, f, start = a
    c.table[0, 2], c.table[1, 1] = c.n_pages, -1
    c.d_table = _i32(c.table)
    before = c.host()
    mb.cache_append(q, k, v, q_out, c.k, c.v, c.d_table, c.d_kv, q_gain=gains[0], k_gain=gains[1], inv_freq=f)
    torch.cuda.synchronize()
    _check_append(case, *a, before)


def _reorder_case(rng, B, n_rows, M, ps, H, D, t, layout, L, spare, beams=False):
    lens = rng.integers(0, M * ps + 1, B)
    lens[:min(B, 3)] = [0, ps, min(ps + 1, M * ps)][:min(B, 3)]
    c = Cache(rng, lens, ps, H, D, t, layout, L, spare=spare, stale=False, max_pages=M)
    src = rng.integers(-1, B + (0 if beams else 1), n_rows)
    if beams:
        src = np.abs(src) % B
    held = np.where((src >= 0) & (src < B), lens[np.clip(src, 0, B - 1)], 0)
    keep = np.where(rng.random(n_rows) < 0.7, held, rng.integers(0, held + 1))
    want = keep + rng.integers(-2, 2 * ps, n_rows)
    return c, src.astype(np.int32), keep.astype(np.int32), want.astype(np.int32)


REORDER = [  # rows, new rows, entries per row, page, H, D, type, layout, layers, spare pages
    (6, 6, 5, 16, 2, 64, "bf16", 0, 3, 40), (6, 9, 5, 16, 2, 64, "bf16", 1, 2, 40), (1, 1, 1, 16, 1, 16, "bf16", 0, 1, 1),
    (8, 3, 4, 32, 1, 128, "f32", 0, 2, 2), (5, 30, 6, 16, 2, 64, "bf16", 0, 1, 4),   # more than there is
    (40, 50, 7, 16, 1, 16, "f32", 1, 2, 200), (3, 1100, 2, 16, 1, 16, "bf16", 0, 1, 3000),
    (70, 70, 300, 16, 1, 16, "bf16", 0, 1, 400), (2, 4096, 1, 16, 1, 16, "bf16", 0, 1, 4096),
    (20, 512, 3, 16, 1, 16, "bf16", 1, 1, 1000), (20, 513, 3, 32, 2, 16, "f32", 1, 2, 1000), (300, 40, 1700, 16, 1, 16, "bf16", 0, 1, 10),
    (9, 9, 4, 16, 1, 16, "bf16", 1, 2, 16500)]


@pytest.mark.parametrize("case", REORDER, ids=lambda c: "-".join(map(str, c)))
def test_reorder(case):
    import torch
    print("case reorder", case, flush=True)
    for seed in range(3):
        rng = np.random.default_rng(seed)
        c, src, keep, want = _reorder_case(rng, *case, beams=seed == 2)
        if seed == 1 and c.table.shape[1] > 1:
            c.table[0, 0] = -1                                    # holes stay holes
            c.table[-1, -1] = c.n_pages + 3
            c.d_table = _i32(c.table)
        k, v = c.host()
        new = torch.full((len(src), c.table.shape[1]), 77, dtype=torch.int32, device="cuda")
        missing = _i32([-1])
        args = (c.d_table, _i32(src), _i32(keep), _i32(want), new, missing)
        mb.cache_reorder(c.k, c.v, *args, page_layout=c.layout)
        wk, wv, wt, wm = ref.cache_reorder(k, v, c.table, src, keep, want, c.layout)
        assert np.array_equal(new.cpu().numpy(), wt), np.argwhere(new.cpu().numpy() != wt)[:4]
        assert int(missing) == wm
        assert np.array_equal(_np(c.k), wk) and np.array_equal(_np(c.v), wv)
        mb.cache_reorder(c.k, c.v, *args, page_layout=c.layout)      # the same call again changes nothing
        assert np.array_equal(new.cpu().numpy(), wt) and np.array_equal(_np(c.k), wk)


def test_reorder_from_no_rows():
    """An empty table: prompts get their first pages."""
    import torch
    k = torch.zeros((1, 10, 16, 1, 16), device="cuda")
    v, table = torch.zeros_like(k), torch.empty((0, 4), dtype=torch.int32, device="cuda")
    new, missing = torch.zeros((3, 4), dtype=torch.int32, device="cuda"), _i32([5])
    mb.cache_reorder(k, v, table, _i32([-1, 0, 7]), _i32([9, 9, 9]), _i32([17, 0, 64]), new, missing)
    assert new.tolist() == [[0, 1, -1, -1], [-1] * 4, [2, 3, 4, 5]] and int(missing) == 0


@pytest.mark.parametrize("M", [1, 63, 64, 65, 129, 300])
def test_pages_of_every_number_of_rows(M):
    """Reordering and compaction of 1 to 35 rows: few rows are shared by several waves, and
    rows of any length end inside a wave's entries."""
    import torch
    for B in (1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 35):
        print("case rows", B, M, flush=True)
        rng = np.random.default_rng(B)
        c, src, keep, want = _reorder_case(rng, B, B, M, 16, 1, 16, "bf16", 0, 1, 3 * B)
        k, v = c.host()
        new, n = torch.full((B, M), 77, dtype=torch.int32, device="cuda"), _i32([-1])
        mb.cache_reorder(c.k, c.v, c.d_table, _i32(src), _i32(keep), _i32(want), new, n)
        k, v, wt, wn = ref.cache_reorder(k, v, c.table, src, keep, want)
        assert np.array_equal(new.cpu().numpy(), wt) and int(n) == wn
        assert np.array_equal(_np(c.k), k) and np.array_equal(_np(c.v), v)
        out = torch.full_like(new, 77)
        mb.cache_compact(c.k, c.v, new, out, n)
        k, v, wt, wn = ref.cache_compact(k, v, wt)
        assert np.array_equal(out.cpu().numpy(), wt) and int(n) == wn
        assert np.array_equal(_np(c.k), k) and np.array_equal(_np(c.v), v)


COMPACT = [  # rows, entries, page, H, D, type, layout, layers, pages of the pool, share held
    (4, 6, 16, 2, 64, "bf16", 0, 3, 30, 0.5), (4, 6, 16, 2, 64, "f32", 1, 2, 24, 0.9), (1, 1, 16, 1, 16, "bf16", 0, 1, 1, 1.0),
    (3, 3, 32, 1, 128, "bf16", 0, 1, 64, 0.0), (8, 8, 16, 1, 16, "bf16", 0, 1, 64, 1.0), (50, 64, 16, 1, 16, "bf16", 0, 2, 3300, 0.4),
    (200, 40, 16, 1, 16, "f32", 0, 1, 40000, 0.7),
    (30, 40, 16, 2, 16, "bf16", 1, 2, 16384, 0.9), (30, 40, 16, 2, 16, "bf16", 1, 2, 16385, 0.9), (700, 100, 16, 1, 16, "bf16", 0, 1, 16000, 0.2),
    (2, 600, 16, 1, 16, "bf16", 0, 1, 1024, 0.85)]


@pytest.mark.parametrize("case", COMPACT, ids=lambda c: "-".join(map(str, c)))
def test_compact(case):
    import torch
    B, M, ps, H, D, t, layout, L, n_pages, share = case
    print("case compact", case, flush=True)
    for seed in range(2):
        rng = np.random.default_rng(seed)
        page = (H, ps, D) if layout else (ps, H, D)
        k, kh = _rand(rng, (L, n_pages) + page, t)
        v, vh = _rand(rng, (L, n_pages) + page, t)
        table = np.full(B * M, -1, np.int32)
        n = min(n_pages, int(share * B * M))
        table[rng.permutation(B * M)[:n]] = rng.permutation(n_pages)[:n]
        if n > 4:
            table[rng.integers(0, B * M, 3)] = [table.max(), -9, n_pages]      # a shared page, two holes
        table = table.reshape(B, M)
        new, used = torch.full((B, M), 5, dtype=torch.int32, device="cuda"), _i32([-4])
        mb.cache_compact(k, v, _i32(table), new, used, page_layout=layout)
        wk, wv, wt, wn = ref.cache_compact(kh, vh, table)
        assert np.array_equal(new.cpu().numpy(), wt) and int(used) == wn
        assert np.array_equal(_np(k), wk) and np.array_equal(_np(v), wv)


def _serve(t, layout, stream=None):
    """A translated context stored, a prompt, decoding, a fork into beams, an end,
    a squeeze, more decoding; checked against attention over dense copies."""
    import torch
    rng = np.random.default_rng(21)
    L, H, Hq, D, ps, n_pages, M = 2, 2, 6, 64, 16, 40, 8
    shape = (L, n_pages) + ((H, ps, D) if layout else (ps, H, D))
    k, v = (torch.full(shape, float("nan"), dtype=_dt(t), device="cuda") for _ in range(2))
    f = torch.from_numpy((100.0 ** -(np.arange(32) / 32)).astype(np.float32)).cuda()
    gain = (1 + 0.1 * torch.randn((L, D), device="cuda")).to(_dt(t))
    dense = {}                                    # row -> list of (k, v) [L][H][D] per position, float64
    table = torch.empty((0, M), dtype=torch.int32, device="cuda")
    lens = []

    def reorder(source, keep, want):
        nonlocal table, dense, lens
        new, missing = torch.empty((len(source), M), dtype=torch.int32, device="cuda"), _i32([0])
        mb.cache_reorder(k, v, table, _i32(source), _i32(keep), _i32(want), new, missing, page_layout=layout)
        assert int(missing) == 0
        table = new
        dense = {b: list(dense[s][:n]) if s >= 0 else [] for b, (s, n) in enumerate(zip(source, keep))}
        lens = list(want)

    def step(counts, turn=True):
        """`counts` new tokens of each row, at the ends of their lengths."""
        n = sum(counts)
        start = _i32(np.concatenate([[0], np.cumsum(counts)]))
        q, kn, vn = (torch.from_numpy(rng.standard_normal((L, n, h, D)).astype(np.float32)).cuda().to(_dt(t)) for h in (Hq, H, H))
        kv = _i32(lens)
        qr = torch.empty_like(q)
        mb.cache_append(q, kn, vn, qr, k, v, table, kv, new_start=start, max_new=max(counts), q_gain=gain if turn else None,
                        k_gain=gain if turn else None, inv_freq=f if turn else None, page_layout=layout)
        outs = []
        for l in range(L):
            o = torch.full_like(q[l], KEEP)
            mb.paged_attention(qr[l], k[l], v[l], table, kv, o, new_start=start, max_new=max(counts), page_layout=layout)
            outs.append(o)
        at = 0
        for b, c in enumerate(counts):
            for i in range(c):
                pos = lens[b] - c + i
                assert len(dense[b]) == pos
                rows = np.stack([[ref._ready(_np(kn[l, at + i, h]), _np(gain[l]) if turn else None, 1e-6,
                                             _np(f) if turn else None, pos, False) for h in range(H)] for l in range(L)])
                rows = torch.from_numpy(rows).to(_dt(t)).double().numpy()
                dense[b].append((rows, _np(vn[:, at + i])))
            for i in range(c):
                pos = lens[b] - c + i
                for l in range(L):
                    K = np.stack([x[0][l] for x in dense[b][:pos + 1]])
                    V = np.stack([x[1][l] for x in dense[b][:pos + 1]])
                    for h in range(Hq):
                        x = K[:, h // 3] @ _np(qr[l, at + i, h]) / 8.0
                        p = np.exp(x - x.max())
                        p /= p.sum()
                        want, mag = p @ V[:, h // 3], p @ np.abs(V[:, h // 3])
                        # the cached keys may differ from the oracle's by a rounding step: a score by
                        # at most eps(t) sum |q k|, the weights by twice that
                        s = (np.abs(K[:, h // 3]) @ np.abs(_np(qr[l, at + i, h]))).max() / 8.0
                        bound = _bound(t, want, mag, s, D, pos + 1) + 4 * HALF[t] * s * mag
                        assert (np.abs(_np(outs[l][at + i, h]) - want) <= bound).all(), (b, pos, l, h)
            at += c

    reorder([-1, -1], [0, 0], [37, 18])
    step([37, 18], turn=False)                    # translated contexts, stored as they are
    reorder([0, 1], [37, 18], [41, 27])
    step([4, 9])                                  # prompts
    reorder([0, 0, 0, 1], [41, 41, 41, 27], [42, 42, 42, 28])
    step([1, 1, 1, 1])                            # three beams and the other conversation
    reorder([2, 0, 2], [42, 42, 42], [43, 43, 43])
    step([1, 1, 1])                               # the other has ended; beams change parents
    new, used = torch.empty_like(table), _i32([0])
    mb.cache_compact(k, v, table, new, used, page_layout=layout)
    assert int(used) == len(set(table[table >= 0].tolist())) and int(new.max()) == int(used) - 1
    table = new
    reorder([0, 1, 2], [43, 20, 43], [44, 25, 44])   # one is cut back and goes on otherwise
    step([1, 5, 1])


@pytest.mark.parametrize("t,layout", [("bf16", 0), ("f32", 1)])
def test_serving_run(t, layout):
    _serve(t, layout)


def test_serving_run_on_another_stream():
    import torch
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _serve("bf16", 0)
    s.synchronize()


def test_graph_of_a_decoding_step():
    """Append, attention (cut), reordering and compaction captured into a graph and
    replayed with new data and lengths, against the eager calls, other work between."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    B, H, Hq, D, ps, M = 3, 2, 12, 128, 16, 128
    n_pages = B * M + 20
    pools = [torch.randn((1, n_pages, ps, H, D), generator=g, device="cuda").bfloat16() for _ in range(2)]
    twin = [p.clone() for p in pools]
    table = torch.randperm(n_pages, generator=g, device="cuda").int()[:B * M].reshape(B, M)
    kv, src, keep = _i32([5, 600, 2000]), _i32([0, 2, 1]), _i32([5, 2000, 333])
    fused = torch.randn((B, 1, Hq + 2 * H, D), generator=g, device="cuda").bfloat16()
    f = torch.rand(D // 2, generator=g, device="cuda")
    a, b = ({"q": torch.empty((B, 1, Hq, D), device="cuda").bfloat16(), "o": torch.empty((B, 1, Hq, D), device="cuda").bfloat16(),
             "t": torch.empty_like(table), "m": _i32([0]), "t2": torch.empty_like(table), "u": _i32([0])} for _ in range(2))

    def step(p, x):
        mb.cache_append(fused[:, :, :Hq], fused[:, :, Hq:Hq + H], fused[:, :, Hq + H:], x["q"], p[0][0], p[1][0], table, kv, inv_freq=f)
        mb.paged_attention(x["q"], p[0][0], p[1][0], table, kv, x["o"])
        mb.cache_reorder(*p, table, src, keep, kv, x["t"], x["m"])
        mb.cache_compact(*p, x["t"], x["t2"], x["u"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(pools, a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pools, a)
    for i in range(4):
        fused.copy_(torch.randn(fused.shape, generator=g, device="cuda"))
        kv.copy_(_i32([6 + i, 601 - 50 * i, 1999 + 3 * i]))
        keep.copy_(_i32([5 - i, 1990 + i, 300 + 17 * i]))
        for p, w in zip(pools, twin):
            p.copy_(w)
        graph.replay()
        torch.cuda.synchronize()
        step(twin, b)
        (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
        for n in a:
            assert torch.equal(a[n], b[n]), (i, n)
        assert all(torch.equal(p, w) for p, w in zip(pools, twin)), i


def test_graph_of_a_large_pool():
    """Reordering and compaction of a pool too large for one launch, captured with a workspace
    of the graph's own and replayed with new rows, other work between."""
    import torch
    rng = np.random.default_rng(8)
    B, M, n_pages = 30, 20, 20000
    c = Cache(rng, rng.integers(0, M * 16 + 1, B).tolist(), 16, 1, 16, "bf16", L=1, stale=False, max_pages=M, spare=n_pages)
    assert mb.cache_workspace_bytes(c.k, c.v, c.d_table, B) > 0
    pools, first = (c.k, c.v), (c.k.clone(), c.v.clone())
    src, keep, want = (_i32(np.zeros(B)) for _ in range(3))
    out = [torch.empty_like(c.d_table) for _ in range(2)] + [_i32([0]), _i32([0])]

    def step(new, packed, missing, used):
        mb.cache_reorder(*pools, c.d_table, src, keep, want, new, missing)
        mb.cache_compact(*pools, new, packed, used)

    step(*out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*out)
    for i in range(4):
        s = rng.integers(-1, B, B)
        k = np.where(s >= 0, np.minimum(np.array(c.kv)[s], rng.integers(0, M * 16 + 1, B)), 0)
        src.copy_(_i32(s)), keep.copy_(_i32(k)), want.copy_(_i32(k + rng.integers(0, 40, B)))
        got = []
        for run in (graph.replay, lambda: step(*out)):
            for p, f in zip(pools, first):
                p.copy_(f)
            for x in out:
                x.fill_(-7)
            run()
            torch.cuda.synchronize()
            (torch.randn(500, 500, device="cuda") @ torch.randn(500, 500, device="cuda")).sum().item()
            got.append([x.clone() for x in (*out, *pools)])
        assert all(torch.equal(a, b) for a, b in zip(*got)), i
        wk, wv, wt, wm = ref.cache_reorder(_np(first[0]), _np(first[1]), c.table, _np(src).astype(int), _np(keep).astype(int), _np(want).astype(int))
        wk, wv, wp, wn = ref.cache_compact(wk, wv, wt)
        assert np.array_equal(out[0].cpu().numpy(), wt) and np.array_equal(out[1].cpu().numpy(), wp)
        assert int(out[2]) == wm and int(out[3]) == wn and np.array_equal(_np(c.k), wk) and np.array_equal(_np(c.v), wv)


def test_binding_refuses():
    """What the binding sees in the tensors: types, devices, shapes, strides."""
    import torch
    rng = np.random.default_rng(0)
    c = Cache(rng, [20, 9], 16, 2, 64, "bf16")
    q, _ = _rand(rng, (2, 3, 4, 64), "bf16")
    o = torch.empty_like(q)
    good = dict(q=q, k_pages=c.k, v_pages=c.v, table=c.d_table, kv_len=c.d_kv, o=o)
    for change in (dict(q=q.float()), dict(q=q[:, :, :, :32]), dict(q=q[:1]), dict(q=q[0]), dict(o=o[:, :2]), dict(o=o.cpu()),
                   dict(k_pages=c.k.float()), dict(k_pages=c.k.half(), v_pages=c.v.half()), dict(v_pages=c.v[:-1]),
                   dict(k_pages=c.k.transpose(1, 2), v_pages=c.v.transpose(1, 2)), dict(table=c.d_table.long()),
                   dict(table=c.d_table[:, ::2]), dict(kv_len=c.d_kv[:1]), dict(kv_len=c.d_kv.cpu()), dict(max_new=2),
                   dict(new_start=_i32([0, 3])), dict(scale=-1.0), dict(scale=1e-50), dict(scale=1e60), dict(window=-1),
                   dict(window=1 << 31), dict(max_kv=1 << 40), dict(o=q), dict(q=q.transpose(2, 3)),
                   dict(o=o[:, :, :1].expand(2, 3, 4, 64)), dict(k_pages=c.k[None], v_pages=c.v[None]),
                   dict(scratch=torch.empty(64))):
        with pytest.raises(mb.MotError):
            mb.paged_attention(**{**good, **change})
    k = q[:, :, :2].contiguous()
    good = dict(q=q, k=k, v=k.clone(), q_out=o, k_pages=c.k, v_pages=c.v, table=c.d_table, kv_len=c.d_kv)
    f = torch.ones(32, device="cuda")
    for change in (dict(q_out=None), dict(v=None), dict(k=None), dict(q=None, q_out=None, k=None, v=None), dict(k=q), dict(k=k[:, :2]),
                   dict(inv_freq=f.double()), dict(inv_freq=f[:4]), dict(inv_freq=torch.ones(64, device="cuda")), dict(inv_freq=f[:0]),
                   dict(q_gain=f.bfloat16()), dict(k_gain=torch.ones(64, device="cuda")), dict(positions=_i32([1, 2])),
                   dict(eps=-1.0), dict(eps=1e60), dict(q_out=q.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :2])):
        with pytest.raises(mb.MotError):
            mb.cache_append(**{**good, **change})
    new, one = torch.empty_like(c.d_table), _i32([0])
    for change in (dict(new_table=new[:1]), dict(new_table=c.d_table), dict(missing=_i32([0, 0])), dict(keep=_i32([1])),
                   dict(workspace=torch.empty(16, dtype=torch.uint8)), dict(source=_i32([0, 1]).long())):
        with pytest.raises(mb.MotError):
            mb.cache_reorder(**{**dict(k_pages=c.k, v_pages=c.v, table=c.d_table, source=_i32([0, 1]), keep=_i32([1, 1]),
                                       want=_i32([1, 1]), new_table=new, missing=one), **change})
    for change in (dict(new_table=new[:1]), dict(used=one.long()), dict(new_table=c.d_table)):
        with pytest.raises(mb.MotError):
            mb.cache_compact(**{**dict(k_pages=c.k, v_pages=c.v, table=c.d_table, new_table=new, used=one), **change})
