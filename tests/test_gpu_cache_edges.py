"""The paged cache at the edges of what its entry points allow, on the GPU against
the float64 oracle: how exact the probabilities are, windows and lengths at the
ends of their ranges, values that are not finite in contexts that are cut, calls
of very many sequences, rows that end.

Bounds are those of test_gpu_cache.py unless a test says otherwise.
"""
from types import SimpleNamespace

import numpy as np
import pytest

from oracle import cache as ref
from paper_2607_28979_amd import binding as mb

from test_gpu_cache import HALF, KEEP, Cache, _attend, _bound, _dt, _i32, _np, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,new,Hq,H,D,cut", [
    ([60, 33, 200], 1, 28, 4, 128, False), ([1500, 90], 1, 12, 2, 128, True), ([150, 77], 4, 14, 2, 64, False),
    ([100, 300, 40], [3, 10, 0], 14, 2, 64, False), ([100, 300, 40], [3, 11, 0], 14, 2, 64, False), ([2000] + [50] * 7, [40] + [1] * 7, 8, 2, 64, True)])
def test_probabilities_of_few_rows(kv, new, Hq, H, D, cut):
    """Tiles of 32 rows: a probability is off by 2^-15 of itself at most (two bf16 terms, the first cut to 8
    bits, 2^-7 of it at most, the second's rounding 2^-8 of that), so the result by 2^-15 of sum of
    softmax |v| beside its own rounding and the fp32 steps.  14 tokens of 7 query heads are 98 rows, more than the 32 of each of 3 sequences: those
    probabilities are rounded once, and the bound is that of tiles of 128 rows."""
    import torch
    rng = np.random.default_rng(sum(kv))
    c = Cache(rng, kv, 16, H, D, "bf16", max_pages=256 if cut else None)
    packed = isinstance(new, list)
    q, _ = _rand(rng, ((sum(new),) if packed else (len(kv), new)) + (Hq, D), "bf16")
    start = np.concatenate([[0], np.cumsum(new)]) if packed else None
    o = torch.full_like(q, KEEP)
    print("case probabilities", kv, new, cut, flush=True)
    mb.paged_attention(q, c.k, c.v, c.d_table, c.d_kv, o, new_start=None if start is None else _i32(start))
    flat = (int(np.prod(q.shape[:-2])), Hq, D)
    want, mag, smax = ref.paged_attention(_np(q).reshape(flat), *c.host(), c.table, c.kv, np.full(flat, KEEP), start,
                                          flat[0] if packed else new)
    most = flat[0] if packed else new
    few = most * (Hq // H) <= 32 or flat[0] * (Hq // H) <= 32 * len(kv)
    assert few == (new != [3, 11, 0])
    bound = HALF["bf16"] * np.abs(want) + mag * (2.0 ** -15 + (2 * (D + 4) * smax + 2 * (max(kv) + 8)) * 2.0 ** -24) + 1e-30
    if not few:
        bound = _bound("bf16", want, mag, smax, D, max(kv), True)
    bad = ~(np.abs(_np(o).reshape(flat) - want) <= bound)
    assert not bad.any(), (int(bad.sum()), bad.size)


@pytest.mark.parametrize("t,n,Hq,D", [("bf16", 3, 6, 64), ("bf16", 30, 4, 64), ("bf16", 30, 28, 128), ("f32", 30, 4, 64), ("f32", 7, 2, 128)])
def test_windows_longer_than_the_context(t, n, Hq, D):
    """A window as long as an int goes is no window, also where new tokens lie at negative
    positions (more of them than positions); so is one of all positions of a table's row, one more,
    one less."""
    import torch
    rng = np.random.default_rng(n)
    kv = [20, 1, 28, 0, 2]
    print("case windows", t, n, flush=True)
    for wide in (None, 256):
        c = Cache(rng, kv, 16, 2, D, t, max_pages=wide)
        most = c.table.shape[1] * 16
        q, _ = _rand(rng, (5, n, Hq, D), t)
        none = _attend(c, q)
        for w in (2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30, most + 1, most, most - 1):
            assert torch.equal(_attend(c, q, window=w), none), (w, most)


@pytest.mark.parametrize("spare", [40, 17000])
def test_rows_that_end_hold_no_page(spare):
    """Beams go on from their parents for many steps in a pool that has no page to lose, and half of
    them end on the way: source -1 and want 0 leaves a row without pages, whatever keep says, and none
    is ever missing."""
    import torch
    rng = np.random.default_rng(spare)
    B, ps = 8, 16
    c = Cache(rng, [50] * B, ps, 1, 16, "bf16", L=1, spare=spare, stale=False, max_pages=6)
    table, live, at = c.table, np.ones(B, bool), 50
    for step in range(40):
        if step in (3, 9, 20, 21):
            live[rng.choice(np.flatnonzero(live))] = False
        parents = np.flatnonzero(live)
        src = np.where(live, rng.choice(parents, B), -1)
        keep, want = np.full(B, at), np.where(live, at + 1, 0)
        new, missing = torch.full((B, 6), 77, dtype=torch.int32, device="cuda"), _i32([-1])
        k, v = c.host()
        mb.cache_reorder(c.k, c.v, _i32(table), _i32(src), _i32(keep), _i32(want), new, missing)
        wk, wv, wt, wm = ref.cache_reorder(k, v, table, src, keep, want)
        new = new.cpu().numpy()
        assert np.array_equal(new, wt) and int(missing) == wm == 0
        assert np.array_equal(_np(c.k), wk) and np.array_equal(_np(c.v), wv)
        assert (new[~live] == -1).all() and (new[live, :-(-(at + 1) // ps)] >= 0).all()
        table, live, at = new, src >= 0, at + 1


@pytest.mark.parametrize("B,n,Hq,H,D,t", [(1, 1, 6, 2, 64, "bf16"), (70, 1, 4, 1, 128, "bf16"), (1, 37, 6, 2, 64, "bf16"),
                                          (70, 37, 4, 1, 128, "bf16"), (1, 1, 6, 2, 64, "f32"), (66, 1, 4, 2, 64, "f32")])
def test_positions_to_the_end_of_the_range(B, n, Hq, H, D, t):
    """One sequence of nearly 2^30 positions, nearly all of them holes, alone and among short ones: its
    blocks are more than 32 bits hold for all sequences and heads, and it is still cut."""
    import torch
    ps, M, kv0 = 1024, 1 << 20, (1 << 30) - 7
    print("case far", B, n, t, flush=True)
    rng = np.random.default_rng(B + n)
    held = np.array([0, 3, 65537, 999999, M - 1])                # entries of the long row that are pages
    k, v = (_rand(rng, (len(held) + B, ps, H, D), t)[0] for _ in range(2))
    pages = rng.permutation(len(held) + B)
    table = torch.full((B, M), -1, dtype=torch.int32, device="cuda")
    long = B // 2
    table[long, torch.from_numpy(held).cuda()] = _i32(pages[:len(held)])
    lens = rng.integers(1, 200, B)
    lens[long] = kv0
    for b in range(B):
        if b != long:
            table[b, 0] = int(pages[len(held) + b])
    q, _ = _rand(rng, (B, n, Hq, D), t)
    o = torch.full_like(q, KEEP)
    mb.paged_attention(q, k, v, table, _i32(lens), o)
    torch.cuda.synchronize()
    pos = torch.from_numpy((held[:, None] * ps + np.arange(ps)[None]).reshape(-1)).cuda()
    for b in sorted({0, long, B - 1}):
        at = pos if b == long else torch.arange(ps, device="cuda")
        ids = torch.from_numpy(pages[:len(held)]).cuda() if b == long else pages[len(held) + b:len(held) + b + 1]
        K, V = (x[ids].reshape(-1, H, D).double() for x in (k, v))
        for h in range(Hq):
            u = int(lens[b]) - n + torch.arange(n, device="cuda")
            s = (q[b, :, h].double() @ K[:, h * H // Hq].T) / D ** 0.5
            s.masked_fill_(at[None] > u[:, None], -float("inf"))
            p = torch.nan_to_num(torch.softmax(s, -1))            # a token at a negative position sees none
            want, mag = p @ V[:, h * H // Hq], p @ V[:, h * H // Hq].abs()
            smax = (q[b, :, h].double().abs() @ K[:, h * H // Hq].abs().T).amax() / D ** 0.5
            bound = _bound(t, _np(want), _np(mag), float(smax), D, len(held) * ps, t == "bf16" and n * Hq // H > 32)
            assert (np.abs(_np(o[b, :, h]) - _np(want)) <= bound).all(), (b, h)


def test_many_sequences_a_loose_bound_and_a_wide_table():
    """512 sequences, 4096 rows of tokens, no bound on a sequence's: the one of 9000 positions is cut."""
    import torch
    rng = np.random.default_rng(9)
    B = 512
    counts = rng.integers(0, 2, B)
    counts[[0, 300, B - 1]] = 1, 3, 5
    kv = counts + rng.integers(0, 20, B)
    kv[300] = 9000
    c = Cache(rng, kv.tolist(), 16, 8, 64, "bf16", stale=False, max_pages=2048)
    q, _ = _rand(rng, (4096, 32, 64), "bf16")
    print("case wide", flush=True)
    whole = _attend(c, q, counts.tolist(), scratch=False)
    cut = _attend(c, q, counts.tolist())
    assert (cut[int(counts.sum()):] == KEEP).all() and not torch.equal(whole, cut)


def _kernels(call):
    """Nodes of the graph that `call` is captured into."""
    import ctypes
    import torch
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call()
    n = ctypes.c_size_t(0)
    hip = ctypes.CDLL(next(iter(mb._hip_runtimes())))
    assert hip.hipGraphGetNodes(ctypes.c_void_p(g.raw_cuda_graph()), None, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("t,B,n,D", [("bf16", 2000, 1, 128), ("bf16", 1500, 9, 64), ("f32", 1300, 4, 64), ("bf16", 65535, 1, 64)])
def test_many_short_sequences_are_one_launch(t, B, n, D):
    """Calls that cut nothing take any number of sequences at once, with the bits of calls of some each."""
    import torch
    rng = np.random.default_rng(B)
    print("case short", t, B, n, flush=True)
    c = Cache(rng, [5, 3, 40, 0], 16, 2, D, t, stale=False)
    pick = rng.integers(0, 4, B)
    table, kv = _i32(c.table[pick]), _i32(np.array(c.kv)[pick])
    q, _ = _rand(rng, (B, n, 8, D), t)
    o = torch.full_like(q, KEEP)
    assert _kernels(lambda: mb.paged_attention(q, c.k, c.v, table, kv, o)) == 1
    parts = torch.full_like(q, KEEP)
    for at in range(0, B, 500):
        m = slice(at, min(at + 500, B))
        mb.paged_attention(q[m], c.k, c.v, table[m], kv[m], parts[m])
    assert torch.equal(o, parts) and (o[:, :] != KEEP).all()
    some = [int(np.flatnonzero(pick == i)[-1]) for i in range(4)]
    few = SimpleNamespace(k=c.k, v=c.v, layout=0, host=c.host, table=c.table[pick[some]], kv=[c.kv[i] for i in pick[some]],
                          d_table=table[some].contiguous(), d_kv=kv[some].contiguous())
    assert torch.equal(_attend(few, q[some].contiguous()), o[some])


@pytest.mark.parametrize("packed", [False, True])
def test_append_of_more_tokens_than_two_to_a_workgroup(packed):
    """2^25 new tokens and some, of one narrow head: more than 2^24 workgroups of two tokens."""
    import torch
    n, ps = (1 << 25) + 37, 1024
    pages = -(-n // ps)
    g = torch.Generator(device="cuda").manual_seed(4)
    print("case far append", packed, flush=True)
    x = torch.randint(-9, 9, (n, 2, 16), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    kp, vp = (torch.full((pages + 2, ps, 1, 16), KEEP, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    order = torch.randperm(pages + 2, generator=g, device="cuda")[:pages].int()
    table = torch.full((3 if packed else 1, pages), -1, dtype=torch.int32, device="cuda")
    table[-1] = order
    k, v = x[:, :1], x[:, 1:]
    if packed:      # no bound, two sequences of none before the one
        mb.cache_append(None, k, v, None, kp, vp, table, _i32([0, 0, n]), new_start=_i32([0, 0, 0, n]))
    else:
        mb.cache_append(None, k[None], v[None], None, kp, vp, table, _i32([n]))
    for pool, y in ((kp, k), (vp, v)):
        assert torch.equal(pool[order.long()].reshape(-1, 1, 16)[:n], y)
        assert int((pool == KEEP).all(-1).sum()) == (pages + 2) * ps - n


def test_append_of_more_rows_than_two_tokens_to_a_workgroup_hold():
    """The same number of queries of 33 heads, whose workgroups take two tokens elsewhere, normed in place:
    rows of twos become the gain exactly (16 of 4 are 64, the mean's root 2, with eps 0)."""
    import torch
    n = (1 << 25) + 37
    print("case far queries", flush=True)
    q = torch.full((1, n, 33, 16), 2.0, dtype=torch.bfloat16, device="cuda")
    gain = torch.arange(-8, 8, device="cuda").bfloat16()
    pool = torch.zeros((1, 16, 1, 16), dtype=torch.bfloat16, device="cuda")
    mb.cache_append(q, None, None, q, pool, pool.clone(), _i32([[0]]), _i32([7]), q_gain=gain, eps=0.0)
    for at in range(0, n, 1 << 21):
        assert (q[0, at:at + (1 << 21)] == gain).all()
    del q
    torch.cuda.empty_cache()


def _poisoned(c, q, counts, window, places):
    """The call's result where (pool, sequence, position, KV head, element, value) are put into the cache: non-finite
    results exactly where and what the definition says, the others within the bound."""
    import torch
    t = "bf16" if q.dtype == torch.bfloat16 else "f32"
    H, D = q.shape[-2:]
    n = q.shape[0] if counts is not None else q.shape[1]
    start = None if counts is None else np.concatenate([[0], np.cumsum(counts)])
    for pool, b, pos, h, d, x in places:
        getattr(c, pool)[c.table[b, pos // c.ps], pos % c.ps, h, d] = x
    outs = []
    for scratch in (None, False):
        o = torch.full_like(q, KEEP)
        mb.paged_attention(q, c.k, c.v, c.d_table, c.d_kv, o, new_start=None if start is None else _i32(start), window=window,
                           scratch=scratch)
        torch.cuda.synchronize()
        outs.append(_np(o).reshape(-1, H, D))
    k, v = c.host()
    flat = np.full(outs[0].shape, KEEP)
    rows = _np(q).reshape(flat.shape)
    with np.errstate(invalid="ignore"):
        want, mag, _ = ref.paged_attention(rows, k, v, c.table, c.kv, flat, start, n, window)
    fine = np.where(np.isfinite(k), k, 0.0)
    smax = ref.paged_attention(rows, fine, np.nan_to_num(v), c.table, c.kv, flat, start, n, window)[2]
    G = H // c.k.shape[2]
    bound = _bound(t, want, mag, smax, D, max(c.kv), t == "bf16" and n * G > 32)
    for got in outs:
        with np.errstate(invalid="ignore"):
            bad = ~((np.abs(got - want) <= bound) & np.isfinite(want)) & (got != want) & ~(np.isnan(got) & np.isnan(want))
        worst = np.unravel_index(np.argmax(bad), bad.shape)
        assert not bad.any(), (int(bad.sum()), worst, got[worst], want[worst], bound[worst])
    return want


@pytest.mark.parametrize("t,n,H,G,D", [("bf16", 1, 2, 6, 128), ("bf16", 1, 2, 7, 64), ("bf16", 3, 2, 4, 128), ("bf16", 40, 2, 4, 64),
                                       ("bf16", 40, 2, 6, 128), ("f32", 1, 2, 6, 64), ("f32", 9, 2, 2, 128), ("f32", 40, 2, 2, 64)])
@pytest.mark.parametrize("window", [0, 1300])
def test_values_that_are_not_finite_in_cut_contexts(t, n, H, G, D, window):
    """NaN and infinite values and keys in the first, a middle and the last part of contexts that are
    cut, some of which only later tokens see or, with a window, only earlier ones."""
    import torch
    print("case poison", t, n, D, window, flush=True)
    for seed in range(3):
        rng = np.random.default_rng(100 * n + seed)
        kv = [2900, 1500, 700 + 3 * n, 40]
        c = Cache(rng, kv, 16, H, D, t, max_pages=1024)
        q, _ = _rand(rng, (len(kv), n, H * G, D), t)
        inf, nan = float("inf"), float("nan")
        low = kv[0] - n - 1300 + 1 + (n > 1)               # the window's low end of the first (or second) token
        places = [[("v", 0, 5, 1, 3, nan), ("v", 1, 1499, 0, 7, -inf)],                     # first part; last position
                  [("v", 0, 1700, 1, 0, inf), ("k", 1, 1500 - n, 0, 1, nan), ("v", 2, 300, 1, 2, inf)],
                  [("v", 0, low, 0, 9, inf), ("v", 1, 1500 - (n + 1) // 2, 1, 4, nan), ("k", 2, 690, 0, 0, nan)]][seed]
        want = _poisoned(c, q, None, window, places)
        assert (~np.isfinite(want)).any() and np.isfinite(want).any()


@pytest.mark.parametrize("t,n,G", [("bf16", 1, 6), ("bf16", 40, 4), ("f32", 9, 2)])
def test_infinite_keys(t, n, G):
    """A key of infinity: its position has all the weight, which is no number, or none of it, by the
    sign of the query's element."""
    print("case infinite keys", t, n, flush=True)
    rng = np.random.default_rng(n)
    for kv, M in (([90, 50], 6), ([2000, 900], 1024)):
        c = Cache(rng, kv, 16, 2, 64, t, max_pages=M)
        q, _ = _rand(rng, (2, n, 2 * G, 64), t)
        want = _poisoned(c, q, None, 0, [("k", 0, 20, 1, 3, float("inf")), ("k", 1, kv[1] - 1, 0, 5, -float("inf"))])
        assert np.isnan(want).any() and np.isfinite(want).any()


@pytest.mark.parametrize("t,n,G,D", [("bf16", 1, 6, 128), ("bf16", 3, 4, 64), ("bf16", 40, 4, 64), ("bf16", 40, 4, 128), ("f32", 9, 2, 64),
                                     ("f32", 20, 2, 128)])
@pytest.mark.parametrize("window", [0, 600])
def test_scores_of_minus_infinity_alone(t, n, G, D, window):
    """Rows all of whose positions have the score -inf have no softmax: NaN, not the zeros of a row that
    sees no position.  Rows that see one other position as well have that one's value."""
    import torch
    print("case minus", t, n, D, window, flush=True)
    rng = np.random.default_rng(n + D)
    for kv, M in (([90, 50, n - 1, 33], 8), ([2000, 900, n - 1, 700], 1024)):
        c = Cache(rng, kv, 16, 2, D, t, max_pages=M)
        q = _rand(rng, (4, n, 2 * G, D), t)[0]
        q[..., 0].abs_()
        for b in (0, 1, 3):                         # KV head 0 of these: nothing but -inf ...
            for j in range(c.kv[b]):
                c.k[c.table[b, j // 16], j % 16, 0, 0] = -float("inf")
        for b, j in ((1, kv[1] - 1), (3, 20)):      # ... but for a position
            c.k[c.table[b, j // 16], j % 16, 0, 0] = 1.0
        want = _poisoned(c, q, None, window, [])
        want = want.reshape(4, n, 2, G, D)
        assert np.isnan(want[0, :, 0]).all() and np.isfinite(want[1, -1]).all() and np.isfinite(want[:, :, 1]).all()
        assert (want[2, 0] == 0).all() and np.isnan(want[1, :-1, 0]).all()


@pytest.mark.parametrize("which,dst_layout,page_layout", [(0, 0, 0), (0, 1, 1), (1, 0, 1), (1, 1, 0), (2, 0, 0), (3, 1, 0)])
def test_answering_from_a_translated_context(which, dst_layout, page_layout):
    """A context translated by mot_translate, stored into pages as it lies (every layer at once), then a
    prompt and single tokens over it, call after call on one stream: the pages hold the translated rows
    bit for bit and every layer's attention is the oracle's over them."""
    import torch
    from paper_2607_28979_amd.configs import WORKLOADS, small_variant
    from paper_2607_28979_amd.inputs import generate
    from helpers import dst_shape, to_dev
    w = small_variant(WORKLOADS[which], L_src=2, L_tgt=3, B=2, T=70).with_(dst_layout=dst_layout)
    t, B, T, H, D, ps = w.dtype, w.B, w.T, w.H_tgt, w.D_tgt, 16
    print("case translated", w.name, dst_layout, page_layout, flush=True)
    inp = generate(w)
    dev = {n: to_dev(getattr(inp, n), t) for n in ("src_k", "src_v", "w1", "b1", "w2", "b2", "wr", "br")}
    dk, dv = (torch.empty(dst_shape(w), dtype=_dt(t), device="cuda") for _ in range(2))
    L, G, M = w.L_tgt, 3, 8
    rng = np.random.default_rng(which)
    table = _i32(rng.permutation(B * M + 3)[:B * M].reshape(B, M))
    shape = (L, B * M + 3) + ((H, ps, D) if page_layout else (ps, H, D))
    k, v = (torch.full(shape, float("nan"), dtype=_dt(t), device="cuda") for _ in range(2))
    f = torch.rand(D // 2, device="cuda")
    mb.translate(dev["src_k"], dev["src_v"], mb.depth_ratio_map(w.L_src, L), dev["w1"], dev["b1"], dev["w2"], dev["b2"], dev["wr"],
                 dev["br"], dk, dv, mb.Shapes.from_workload(w))
    rows = [x.transpose(2, 3) if dst_layout else x for x in (dk, dv)]          # [L][B][T][H][D]
    mb.cache_append(None, *rows, None, k, v, table, _i32([T] * B), page_layout=page_layout)
    steps = []
    for n, kv in ((9, T + 9), (1, T + 10), (1, T + 11)):
        fused = _rand(rng, (L, B, n, G * H + 2 * H, D), t)[0]
        q = torch.empty((L, B, n, G * H, D), dtype=_dt(t), device="cuda")
        mb.cache_append(fused[..., :G * H, :], fused[..., G * H:G * H + H, :], fused[..., G * H + H:, :], q, k, v, table, _i32([kv] * B),
                        inv_freq=f, page_layout=page_layout)
        o = torch.full_like(q, KEEP)
        for l in range(L):
            mb.paged_attention(q[l], k[l], v[l], table, _i32([kv] * B), o[l], page_layout=page_layout)
        steps.append((n, kv, q, o))
    torch.cuda.synchronize()
    for pool, x in ((k, rows[0]), (v, rows[1])):
        held = pool[:, table.long()]                                            # [L][B][M] x page
        held = (held.transpose(3, 4) if page_layout else held).reshape(L, B, M * ps, H, D)
        assert torch.isfinite(x).all() and torch.equal(held[:, :, :T], x)
        assert torch.isfinite(held[:, :, :T + 11]).all() and torch.isnan(held[:, :, T + 11:]).all()
    for n, kv, q, o in steps:
        for l in range(L):
            flat = _np(q[l]).reshape(B * n, G * H, D)
            want, mag, smax = ref.paged_attention(flat, _np(k[l]), _np(v[l]), table.cpu().numpy(), [kv] * B, flat, max_new=n,
                                                  layout=page_layout)
            assert (np.abs(_np(o[l]).reshape(want.shape) - want) <= _bound(t, want, mag, smax, D, kv)).all(), (n, l)


@pytest.mark.parametrize("t,n,G,D", [("bf16", 1, 6, 128), ("bf16", 3, 4, 64), ("bf16", 40, 4, 128), ("f32", 9, 2, 64), ("f32", 1, 2, 128)])
def test_holes_in_cut_contexts(t, n, G, D):
    """Long contexts that are holes throughout, or but for a page, or but for the last position's: rows that see
    nothing are zeros, also where a window leaves them only holes."""
    import torch
    print("case cut holes", t, n, D, flush=True)
    rng = np.random.default_rng(n + G)
    c = Cache(rng, [3000, 2100, 1500, 70], 16, 2, D, t, max_pages=1024)
    c.table[0] = -1
    c.table[1, :60] = c.n_pages
    c.table[1, 61:] = -7
    c.table[2, :93] = -1
    c.d_table = _i32(c.table)
    q, _ = _rand(rng, (4, n, 2 * G, D), t)
    for window in (0, 64, 1200):
        o = _attend(c, q, window=window)
        assert (o[0] == 0).all() and (window != 64 or (o[1] == 0).all())
        assert torch.isfinite(_attend(c, q, window=window, scratch=False)).all()
