"""CPU tests of the paged cache's entry points: what they refuse, before any
launch (addresses here are never dereferenced), the sizes of their workspaces,
the struct layouts, and their float64 oracle on worked cases."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import cache as ref
from paper_2607_28979_amd import binding as mb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000
GIB = 1 << 30


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mb.lib_path()):
        pytest.skip("libmot.so not built (run __graft_entry__.build())")
    return mb.load_library()


def _cache(**kw):
    base = dict(L=1, n_pages=64, page_size=16, H_kv=2, D=64, B=3, max_pages=8, dtype=mb.MOT_BF16, page_layout=0)
    base.update(kw)
    return mb._CacheShapes(**base)


def _rows(heads, D, tokens):
    return mb._Strides(0, tokens * heads * D, heads * D, D)


def _attend(cache=None, ptrs=None, strides=None, **kw):
    c = cache or _cache()
    base = dict(n_new=12, max_new=4, H_q=4, window=0, max_kv=0, scale=0.0, workspace=None, workspace_bytes=0)
    base.update(kw)
    D = c.D
    st = {"q": _rows(base["H_q"], D, base["max_new"]), "o": _rows(base["H_q"], D, base["max_new"]), **(strides or {})}
    s = mb._AttendShapes(*[base[n] for n in ("n_new", "max_new", "H_q", "window", "max_kv", "scale")], st["q"], st["o"],
                         base["workspace"], base["workspace_bytes"])
    p = dict(q=FAKE, k=FAKE + GIB, v=FAKE + 2 * GIB, table=FAKE + 3 * GIB, kv_len=FAKE + 4 * GIB, start=None,
             o=FAKE + 5 * GIB)
    p.update(ptrs or {})
    return mb.STATUS[mb.load_library().mot_paged_attention(
        *[p[n] for n in ("q", "k", "v", "table", "kv_len", "start", "o")], ctypes.byref(c), ctypes.byref(s), None)]


@pytest.mark.parametrize("kw,code", [
    (dict(L=0), "BAD_SHAPE"), (dict(L=2), "BAD_SHAPE"), (dict(n_pages=0), "BAD_SHAPE"), (dict(B=-1), "BAD_SHAPE"),
    (dict(B=65536), "BAD_SHAPE"), (dict(max_pages=0), "BAD_SHAPE"), (dict(H_kv=0), "BAD_SHAPE"), (dict(D=0), "BAD_SHAPE"),
    (dict(dtype=2), "BAD_SHAPE"), (dict(page_layout=2), "BAD_SHAPE"), (dict(page_size=0), "BAD_SHAPE"),
    (dict(page_size=8), "UNSUPPORTED"), (dict(page_size=48), "UNSUPPORTED"), (dict(page_size=2048), "UNSUPPORTED"),
    (dict(D=96), "UNSUPPORTED"), (dict(D=72), "UNSUPPORTED"), (dict(D=256), "UNSUPPORTED"),
    (dict(max_pages=1 << 27), "BAD_SHAPE"), (dict(H_kv=3), "BAD_SHAPE")])
def test_attention_refuses_caches(lib, kw, code):
    assert _attend(cache=_cache(**kw)) == "MOT_ERR_" + code


@pytest.mark.parametrize("kw,code", [
    (dict(n_new=-1), "BAD_SHAPE"), (dict(max_new=-1), "BAD_SHAPE"), (dict(n_new=13), "BAD_SHAPE"),
    (dict(max_new=13), "BAD_SHAPE"), (dict(n_new=1 << 27), "BAD_SHAPE"), (dict(H_q=0), "BAD_SHAPE"),
    (dict(H_q=5), "BAD_SHAPE"), (dict(window=-1), "BAD_SHAPE"), (dict(max_kv=-1), "BAD_SHAPE"),
    (dict(scale=-1.0), "BAD_SHAPE"), (dict(scale=float("nan")), "BAD_SHAPE"), (dict(scale=float("inf")), "BAD_SHAPE")])
def test_attention_refuses_sizes(lib, kw, code):
    assert _attend(**kw) == "MOT_ERR_" + code


@pytest.mark.parametrize("ptrs,code", [
    (dict(q=None), "NULL_ARG"), (dict(v=None), "NULL_ARG"), (dict(table=None), "NULL_ARG"), (dict(kv_len=None), "NULL_ARG"),
    (dict(o=None), "NULL_ARG"), (dict(q=FAKE + 8), "MISALIGNED"), (dict(k=FAKE + GIB + 2), "MISALIGNED"),
    (dict(table=FAKE + 3 * GIB + 2), "MISALIGNED"), (dict(o=FAKE + 16), "BAD_SHAPE"),
    (dict(o=FAKE + GIB + 16), "BAD_SHAPE"), (dict(table=FAKE + 5 * GIB + 4), "BAD_SHAPE"),
    (dict(kv_len=FAKE + 5 * GIB), "BAD_SHAPE")])
def test_attention_refuses_pointers(lib, ptrs, code):
    assert _attend(ptrs=ptrs) == "MOT_ERR_" + code


@pytest.mark.parametrize("name,st,code", [
    ("q", (0, 1024, 256, 60), "MISALIGNED"), ("q", (0, 1024, -256, 64), "BAD_SHAPE"), ("q", (0, 1 << 41, 256, 64), "BAD_SHAPE"),
    ("o", (0, 1024, 256, 0), "BAD_SHAPE"), ("o", (0, 1024, 192, 64), "BAD_SHAPE"), ("o", (0, 1016, 256, 64), "BAD_SHAPE"),
    ("o", (0, 0, 256, 64), "BAD_SHAPE")])
def test_attention_refuses_strides(lib, name, st, code):
    assert _attend(strides={name: mb._Strides(*st)}) == "MOT_ERR_" + code


def test_attention_no_ops(lib):
    assert _attend(n_new=0, max_new=0, ptrs=dict(q=None, o=None)) == "MOT_OK"
    assert _attend(cache=_cache(B=0), n_new=0, max_new=0, ptrs=dict(table=None, kv_len=None)) == "MOT_OK"
    s = mb._AttendShapes(1, 1, 4, 0, 0, 0.0, _rows(4, 64, 1), _rows(4, 64, 1))
    assert mb.load_library().mot_attend_workspace_bytes(ctypes.byref(_cache(D=80)), ctypes.byref(s)) == mb._SIZE_MAX


def test_attention_workspace(lib):
    # a long decoding step is cut, and its workspace is checked where it is used
    c = _cache(B=1, max_pages=2048, H_kv=2)
    s = mb._AttendShapes(1, 1, 4, 0, 0, 0.0, _rows(4, 64, 1), _rows(4, 64, 1))
    need = mb.load_library().mot_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(s))
    assert need > 0 and need % 4 == 0
    free = FAKE + 40 * GIB
    kw = dict(cache=c, n_new=1, max_new=1, workspace_bytes=need)
    assert _attend(workspace=free + 8, **kw) == "MOT_ERR_MISALIGNED"
    for at, n in ((FAKE, 4 * 64 * 2), (FAKE + GIB, 64 * 16 * 128 * 2), (FAKE + 3 * GIB, 2048 * 4), (FAKE + 5 * GIB, 512)):
        assert _attend(workspace=at + n - 16, **kw) == "MOT_ERR_BAD_SHAPE"
        assert _attend(workspace=at - need + 16, **kw) == "MOT_ERR_BAD_SHAPE"


def _append(cache=None, ptrs=None, rope=None, strides=None, **kw):
    c = cache or _cache()
    base = dict(n_new=12, max_new=4, H_q=4, rotary_dim=0, interleaved=0, eps=1e-6)
    base.update(kw)
    st = {"q": _rows(4, c.D, 4), "q_out": _rows(4, c.D, 4), "k": _rows(2, c.D, 4), "v": _rows(2, c.D, 4), **(strides or {})}
    s = mb._AppendShapes(*[base[n] for n in ("n_new", "max_new", "H_q", "rotary_dim", "interleaved", "eps")],
                         st["q"], st["q_out"], st["k"], st["v"])
    names = ("q", "k", "v", "q_out", "k_pages", "v_pages", "table", "kv_len", "start")
    p = {n: FAKE + i * GIB for i, n in enumerate(names)}
    p["start"] = None
    p.update(ptrs or {})
    r = mb._Rope(**(rope or {}))
    return mb.STATUS[mb.load_library().mot_cache_append(*[p[n] for n in names], ctypes.byref(r), ctypes.byref(c),
                                                        ctypes.byref(s), None)]


@pytest.mark.parametrize("kw,code", [
    (dict(n_new=13), "BAD_SHAPE"), (dict(max_new=13), "BAD_SHAPE"), (dict(H_q=0), "BAD_SHAPE"),
    (dict(rotary_dim=8), "BAD_SHAPE"), (dict(rotary_dim=80), "BAD_SHAPE"), (dict(rotary_dim=-16), "BAD_SHAPE"),
    (dict(interleaved=2), "BAD_SHAPE"), (dict(eps=-1.0), "BAD_SHAPE"), (dict(eps=float("nan")), "BAD_SHAPE"),
    (dict(ptrs=dict(q=None)), "NULL_ARG"), (dict(ptrs=dict(q_out=None)), "NULL_ARG"), (dict(ptrs=dict(v=None)), "NULL_ARG"),
    (dict(ptrs=dict(q=None, q_out=None, k=None, v=None)), "NULL_ARG"), (dict(ptrs=dict(table=None)), "NULL_ARG"),
    (dict(ptrs=dict(k_pages=None)), "NULL_ARG"), (dict(ptrs=dict(k=FAKE + 4)), "MISALIGNED"),
    (dict(rope=dict(q_gain=FAKE + 2)), "MISALIGNED"), (dict(rope=dict(inv_freq=FAKE + 2)), "MISALIGNED"),
    (dict(ptrs=dict(v_pages=FAKE + 4 * GIB + 1024)), "BAD_SHAPE"), (dict(ptrs=dict(q_out=FAKE + 16)), "BAD_SHAPE"),
    (dict(ptrs=dict(q_out=FAKE + GIB)), "BAD_SHAPE"), (dict(ptrs=dict(k_pages=FAKE + GIB)), "BAD_SHAPE"),
    (dict(ptrs=dict(q_out=FAKE), strides=dict(q_out=mb._Strides(0, 2048, 256, 64))), "BAD_SHAPE"),
    (dict(strides=dict(q_out=mb._Strides(0, 1024, 64, 64))), "BAD_SHAPE"),
    (dict(strides=dict(k=mb._Strides(0, 512, 128, 4))), "MISALIGNED"),
    (dict(cache=_cache(D=72)), "UNSUPPORTED"), (dict(cache=_cache(D=272)), "UNSUPPORTED"),
    (dict(cache=_cache(page_size=24)), "UNSUPPORTED")])
def test_append_refuses(lib, kw, code):
    assert _append(**kw) == "MOT_ERR_" + code


def test_append_no_ops(lib):
    assert _append(n_new=0, max_new=0, ptrs=dict(q=None, q_out=None, k=None, v=None, table=None)) == "MOT_OK"


def _pages(fn, cache=None, n_rows=3, ws=FAKE + 20 * GIB, ws_bytes=None, **ptrs):
    c = cache or _cache()
    names = ("k", "v", "table", "source", "keep", "want", "new", "count") if fn == "reorder" else ("k", "v", "table", "new", "count")
    p = {n: FAKE + i * GIB for i, n in enumerate(names)}
    p.update(ptrs)
    need = mb.load_library().mot_cache_workspace_bytes(ctypes.byref(c), n_rows if fn == "reorder" else 0)
    nb = need if ws_bytes is None else ws_bytes
    call = getattr(mb.load_library(), "mot_cache_" + fn)
    extra = (n_rows,) if fn == "reorder" else ()
    return mb.STATUS[call(*[p[n] for n in names], ctypes.byref(c), *extra, ws, nb, None)]


@pytest.mark.parametrize("fn", ["reorder", "compact"])
def test_pages_refuse(lib, fn):
    assert _pages(fn, k=None) == "MOT_ERR_NULL_ARG"
    assert _pages(fn, new=None) == "MOT_ERR_NULL_ARG"
    assert _pages(fn, count=None) == "MOT_ERR_NULL_ARG"
    big = _cache(n_pages=20000)      # small ones need no workspace
    assert _pages(fn, cache=big, ws=None) == "MOT_ERR_NULL_ARG"
    assert _pages(fn, cache=big, ws_bytes=64) == "MOT_ERR_WORKSPACE_TOO_SMALL"
    assert _pages(fn, cache=big, ws=FAKE + 20 * GIB + 4) == "MOT_ERR_MISALIGNED"
    assert _pages(fn, cache=big, ws=FAKE + 64) == "MOT_ERR_BAD_SHAPE"
    assert _pages(fn, table=FAKE + 2 * GIB + 1) == "MOT_ERR_MISALIGNED"
    assert _pages(fn, new=FAKE + 2 * GIB) == "MOT_ERR_BAD_SHAPE"           # in place
    assert _pages(fn, v=FAKE + 4096) == "MOT_ERR_BAD_SHAPE"
    assert _pages(fn, count=FAKE) == "MOT_ERR_BAD_SHAPE"
    assert _pages(fn, cache=_cache(page_size=17)) == "MOT_ERR_UNSUPPORTED"
    assert _pages(fn, cache=_cache(L=300)) == "MOT_ERR_BAD_SHAPE"
    if fn == "reorder":
        assert _pages(fn, source=None) == "MOT_ERR_NULL_ARG"
        assert _pages(fn, n_rows=4097) == "MOT_ERR_BAD_SHAPE"
        assert _pages(fn, n_rows=-1) == "MOT_ERR_BAD_SHAPE"
        assert _pages(fn, n_rows=0, k=None) == "MOT_OK"
    else:
        assert _pages(fn, cache=_cache(B=0), k=None) == "MOT_OK"


def test_struct_layouts(tmp_path):
    structs = {"mot_cache_shapes": mb._CacheShapes, "mot_strides": mb._Strides, "mot_attend_shapes": mb._AttendShapes,
               "mot_append_shapes": mb._AppendShapes, "mot_rope": mb._Rope}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "mot.h"', "int main(void) {"]
    for cname, cls in structs.items():
        lines.append('printf("%s size %%zu\\n", sizeof(%s));' % (cname, cname))
        lines += ['printf("%s %s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f) for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]) + "\n")
    subprocess.run(["gcc", "-std=c99", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    "/opt/rocm/include", str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out.splitlines()}
    packed = {"mot_cache_shapes": mb._CACHE, "mot_append_shapes": mb._APPEND, "mot_rope": mb._ROPE}
    for cname, st in packed.items():
        assert st.size == got[(cname, "size")], cname
    assert mb._ATTEND.size == got[("mot_attend_shapes", "workspace")]
    assert mb._ATTEND.size + mb._SCRATCH.size == got[("mot_attend_shapes", "size")]
    for cname, cls in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert got[(cname, f)] == getattr(cls, f).offset, (cname, f)


# the oracle on worked cases --------------------------------------------------------------------------------------

def test_oracle_attention_by_hand():
    """Two positions in two pages, equal keys: the mean of their values; a hole
    leaves one; a window of one leaves the token's own."""
    k = np.zeros((3, 16, 1, 64))
    v = np.zeros((3, 16, 1, 64))
    v[2, 15], v[0, 0] = 1.0, 3.0                    # positions 15 and 16
    v[2, :15] = 1.0
    q = np.ones((1, 1, 64))
    args = lambda t, kv=17, **kw: ref.paged_attention(q, k, v, np.array([t]), np.array([kv]), np.full(q.shape, 9.0),   # noqa: E731
                                                      max_new=1, **kw)[0]
    assert np.allclose(args([2, 0]), (16 * 1 + 3) / 17)
    assert np.allclose(args([-1, 0]), 3) and np.allclose(args([2, 7]), 1)
    assert np.allclose(args([2, 0], window=1), 3) and np.allclose(args([2, 0], window=2), 2)
    assert (args([2, 0], kv=0) == 0).all() and (args([5, 5]) == 0).all()


def test_oracle_append_by_hand():
    k = np.zeros((1, 1, 1, 16))
    k[0, 0, 0, 0] = 2.0
    pool = np.full((1, 2, 16, 1, 16), 7.0)
    f = np.array([np.pi / 8] + [0.0] * 7)
    out = lambda inter: ref.cache_append(None, k, k, None, pool, pool, np.array([[1]]), np.array([5]), max_new=1,     # noqa: E731
                                         inv_freq=f, interleaved=inter)
    _, kp, vp = out(False)
    assert np.allclose(kp[0, 1, 4, 0, [0, 8]], [0, 2]) and vp[0, 1, 4, 0, 0] == 2 and (kp[0, 0] == 7).all()
    _, kp, vp = out(True)
    assert np.allclose(kp[0, 1, 4, 0, :2], [0, 2])
    q = np.full((1, 1, 1, 16), 3.0)
    got = ref.cache_append(q, None, None, q, pool, pool, np.array([[1]]), np.array([0]), max_new=1,
                           q_gain=np.full((1, 16), 5.0), eps=0.0)[0]
    assert np.allclose(got, 5.0)


def test_oracle_reorder_by_hand():
    """Row 0 goes on, row 1 forks from row 0 (whole page shared, last page
    copied), row 2 is empty: its pages are free and go to the rows in order."""
    pool = np.arange(8 * 16, dtype=float).reshape(1, 8, 16, 1, 1)
    table = np.array([[5, 3, -1], [0, -1, -1], [2, 1, -1]])
    k, v, new, missing = ref.cache_reorder(pool, pool, table, [0, 0, -1], [20, 20, 0], [33, 21, 3])
    assert new.tolist() == [[5, 3, 0], [5, 1, -1], [2, -1, -1]] and missing == 0
    assert (k[0, 1, :4] == pool[0, 3, :4]).all() and (k[0, 1, 4:] == pool[0, 1, 4:]).all()
    assert ref.cache_reorder(pool, pool, table, [0, 0, -1], [20, 20, 0], [48, 48, 48])[3] == 0
    assert ref.cache_reorder(pool, pool, table[:, :2], [0] * 9, [20] * 9, [20] * 9)[3] == 2


def test_oracle_compact_by_hand():
    pool = np.arange(6.0).reshape(1, 6, 1, 1, 1)
    k, v, new, n = ref.cache_compact(pool, pool, np.array([[5, 1], [5, -1], [4, 9]]))
    assert n == 3 and new.tolist() == [[2, 1], [2, -1], [0, -1]]
    assert k.ravel().tolist() == [4, 1, 5, 3, 4, 5]


def test_oracle_reorder_of_rows_that_end():
    """A row that ends (source -1, want 0) holds no page and misses none; with want left at
    its length it takes pages anew."""
    pool = np.zeros((1, 4, 16, 1, 1))
    table = np.array([[0, 1, -1], [2, 3, -1]])
    new, missing = ref.cache_reorder(pool, pool, table, [0, -1], [20, 20], [21, 0])[2:]
    assert new.tolist() == [[0, 1, -1], [-1, -1, -1]] and missing == 0
    new, missing = ref.cache_reorder(pool, pool, table, [0, -1], [20, 20], [21, 40])[2:]
    assert new.tolist() == [[0, 1, -1], [2, 3, -1]] and missing == 1


@pytest.mark.parametrize("B,n_new,max_new,H_q,H_kv,D,max_pages,ps,dtype,cut", [
    (512, 4096, 4096, 32, 8, 64, 2048, 16, mb.MOT_BF16, True),      # many sequences, a loose bound on their tokens
    (600, 1000, 1000, 28, 4, 128, 8192, 64, mb.MOT_BF16, True), (70, 70, 1, 2, 2, 64, 1 << 14, 1024, mb.MOT_BF16, True),
    (64, 64, 64, 16, 16, 64, 1 << 14, 1024, mb.MOT_F32, False), (2, 37, 37, 28, 4, 128, 1 << 20, 1024, mb.MOT_BF16, True),
    (20, 64, 64, 16, 16, 64, 1 << 16, 1024, mb.MOT_F32, True)])
def test_long_contexts_are_cut_whatever_the_table_holds(lib, B, n_new, max_new, H_q, H_kv, D, max_pages, ps, dtype, cut):
    """Tables of wide rows, many sequences and loose bounds do not keep a long sequence whole; what does
    (fp32) is as many tiles as fill the chip: up to 64 / 16 + 64 of them on 16 heads are 1088, from 512 on
    nothing is cut."""
    c = _cache(B=B, H_kv=H_kv, D=D, max_pages=max_pages, page_size=ps, dtype=dtype)
    s = mb._AttendShapes(n_new, max_new, H_q, 0, 0, 0.0, _rows(H_q, D, n_new), _rows(H_q, D, n_new))
    need = lib.mot_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(s))
    assert (0 < need < 1 << 30) if cut else need == 0


@pytest.mark.parametrize("cache,kw", [
    (dict(dtype=mb.MOT_F32, B=1, H_kv=16), dict(n_new=1 << 24, max_new=1 << 24, H_q=16)),
    (dict(dtype=mb.MOT_F32, B=1, H_kv=16, max_pages=4096), dict(n_new=1 << 24, max_new=1 << 24, H_q=16)),
    (dict(B=64, H_kv=64), dict(n_new=4 * ((1 << 24) - 8), max_new=1 << 24, H_q=64, packed=True))])
def test_attention_refuses_what_no_launch_holds(lib, cache, kw):
    """More workgroups than a launch takes are found before anything is launched."""
    kw = dict(kw)
    packed = kw.pop("packed", False)
    far = {n: FAKE + i * (1 << 41) for i, n in enumerate(("q", "k", "v", "table", "kv_len", "start", "o"))}
    if not packed:
        far["start"] = None
    assert _attend(cache=_cache(**cache), ptrs=far, **kw) == "MOT_ERR_UNSUPPORTED"


def test_tokens_of_a_call(lib):
    for n in (4 * ((1 << 24) - 8) + 1, 1 << 26):
        for call in (_append, _attend):
            assert call(cache=_cache(B=1), n_new=n, max_new=n) == "MOT_ERR_BAD_SHAPE"
            assert b"2^26" in lib.mot_last_error()


def test_no_cut_that_no_launch_joins(lib):
    """Where the partial sums' rows are more than a launch holds, nothing is cut."""
    c = _cache(B=3, H_kv=1024, max_pages=2048)
    sizes = lambda n, G: mb._AttendShapes(n, n, 1024 * G, 0, 0, 0.0, _rows(1024 * G, 64, n), _rows(1024 * G, 64, n))  # noqa: E731
    need = lambda *a: lib.mot_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(sizes(*a)))  # noqa: E731
    assert need(16, 2) > 0      # 3 sequences, 16 x 2048 rows
    c = _cache(B=65535, H_kv=1024, max_pages=2048)
    assert need(65535, 1) == 0 and need(16, 1) > 0


@pytest.mark.parametrize("scale", [3.0e38, 2.4e38])
def test_attention_refuses_scales_past_fp32(lib, scale):
    """scale * log2(e) is what scores are multiplied by: from 2.36e38 on it is infinite, and rows of
    zeros would be NaN."""
    assert _attend(scale=scale) == "MOT_ERR_BAD_SHAPE"
