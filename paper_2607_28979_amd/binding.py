"""Thin ctypes binding of libmot (argument marshalling only).

Every step of the translation runs in the HIP kernels of ``csrc/libmot.so``.
This module turns torch tensors into device pointers and the current torch
stream into a ``hipStream_t``; it has no compute path of its own and raises
``MotError`` when the library is missing or a call fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(HERE, "csrc", "libmot.so")

MOT_F32, MOT_BF16 = 0, 1
LAYOUT_BTHD, LAYOUT_BHTD = 0, 1
ACT_GELU, ACT_IDENTITY = 0, 1
ALGO_AUTO, ALGO_UNFUSED, ALGO_FUSED, ALGO_ROUTED = 0, 1, 2, 3

STATUS = {0: "MOT_OK", 1: "MOT_ERR_NULL_ARG", 2: "MOT_ERR_BAD_SHAPE", 3: "MOT_ERR_BAD_LAYER_MAP",
          4: "MOT_ERR_UNSUPPORTED", 5: "MOT_ERR_MISALIGNED", 6: "MOT_ERR_WORKSPACE_TOO_SMALL",
          7: "MOT_ERR_HIP"}

EXPORTED = ("mot_translate", "mot_workspace_bytes", "mot_depth_ratio_map", "mot_status_string",
            "mot_last_error", "mot_abi_version", "mot_restore_kv", "mot_topS_select",
            "mot_replay_attention", "mot_backbone_param_count", "mot_backbone_translate",
            "mot_usage_stats", "mot_replay_workspace_bytes", "mot_backbone_workspace_bytes",
            "mot_replay_attention_noalloc", "mot_translate_scratch", "mot_translate_scratch_bytes",
            "mot_paged_attention", "mot_attend_workspace_bytes", "mot_cache_append", "mot_cache_reorder",
            "mot_cache_compact", "mot_cache_workspace_bytes")


class MotError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        self.name = STATUS.get(status, "MOT_ERR_%d" % status)
        super().__init__("%s: %s" % (self.name, detail))


class _Shapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "L_src", "L_tgt", "B", "T", "H_src", "D_src", "H_tgt", "D_tgt", "E", "top_k", "hidden",
        "dtype", "src_layout", "dst_layout", "act", "algo", "streams")] + [
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("usage", ctypes.c_void_p)]


class _RestoreShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("L", "B", "T", "d_act", "H_tgt", "D_tgt", "dtype",
                                             "dst_layout")]


class _BackboneDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("d_h", "n_heads", "d_ff", "n_slots")]


class _ReplayShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "H_q", "H_kv", "D", "S", "kv_layout")] + [
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class _CacheShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("L", "n_pages", "page_size", "H_kv", "D", "B", "max_pages", "dtype",
                                             "page_layout")]


class _Strides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("layer", "batch", "token", "head")]


class _AttendShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_new", "max_new", "H_q", "window", "max_kv")] + [
        ("scale", ctypes.c_float), ("q", _Strides), ("o", _Strides), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t)]


class _AppendShapes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_new", "max_new", "H_q", "rotary_dim", "interleaved")] + [
        ("eps", ctypes.c_float)] + [(n, _Strides) for n in ("q", "q_out", "k", "v")]


class _Rope(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q_gain", "k_gain", "inv_freq", "positions")]


class _TW(ctypes.Structure):
    _fields_ = [("w1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("w2", ctypes.c_void_p),
                ("b2", ctypes.c_void_p)]


class _RW(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("b", ctypes.c_void_p)]


@dataclass
class Shapes:
    L_src: int
    L_tgt: int
    B: int
    T: int
    H_src: int
    D_src: int
    H_tgt: int
    D_tgt: int
    E: int
    hidden: int
    dtype: int = MOT_BF16
    top_k: int = 0            # 0 = E
    src_layout: int = LAYOUT_BTHD
    dst_layout: int = LAYOUT_BTHD
    act: int = ACT_GELU
    algo: int = ALGO_AUTO
    streams: int = 2          # 2 = keys and values; 1 = one activation stream (MoT-h)

    def c(self, workspace=None, workspace_bytes=0, usage=None) -> _Shapes:
        return _Shapes(self.L_src, self.L_tgt, self.B, self.T, self.H_src, self.D_src, self.H_tgt,
                       self.D_tgt, self.E, self.top_k or self.E, self.hidden, self.dtype,
                       self.src_layout, self.dst_layout, self.act, self.algo, self.streams,
                       workspace, workspace_bytes, usage)

    @classmethod
    def from_workload(cls, w, **kw) -> "Shapes":
        return cls(w.L_src, w.L_tgt, w.B, w.T, w.H_src, w.D_src, w.H_tgt, w.D_tgt, w.E, w.hidden,
                   dtype=MOT_F32 if w.dtype == "f32" else MOT_BF16, src_layout=w.src_layout,
                   dst_layout=w.dst_layout, **{"top_k": w.top_k, "streams": w.streams, **kw})


_lib = None
_SIZE_MAX = ctypes.c_size_t(-1).value


def lib_path() -> str:
    return _LIB_PATH


def _hip_runtimes() -> set:
    """Distinct files of the HIP runtime mapped into this process (Linux)."""
    try:
        with open("/proc/self/maps") as f:
            return {os.path.realpath(ln.split()[-1]) for ln in f
                    if "libamdhip64.so" in ln and ln.split()[-1].startswith("/")}
    except OSError:
        return set()


def load_library():
    """Load libmot.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise MotError(-1, "libmot.so not found at %s; build it with "
                               "`python -m paper_2607_28979_amd.build`" % _LIB_PATH)
        # PyTorch for ROCm ships its own HIP runtime.  Loading torch first lets
        # libmot bind to that same runtime (the dynamic linker matches its
        # soname), so streams and device pointers from torch are valid here;
        # loading libmot first would bring a second, separate runtime into
        # the process.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        lib = ctypes.CDLL(_LIB_PATH)
        runtimes = _hip_runtimes()
        if len(runtimes) > 1:
            raise MotError(-1, "two HIP runtimes are loaded in this process (%s); import torch "
                               "before loading libmot" % ", ".join(sorted(runtimes)))
        lib.mot_translate.restype = ctypes.c_int
        lib.mot_translate.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.POINTER(_TW), ctypes.POINTER(_RW), ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.POINTER(_Shapes), ctypes.c_void_p]
        lib.mot_translate_scratch.restype = ctypes.c_int
        lib.mot_translate_scratch.argtypes = lib.mot_translate.argtypes[:8] + [ctypes.c_void_p, ctypes.c_size_t,
                                                                               ctypes.c_void_p]
        lib.mot_translate_scratch_bytes.restype = ctypes.c_size_t
        lib.mot_translate_scratch_bytes.argtypes = [ctypes.POINTER(_Shapes), ctypes.c_void_p]
        lib.mot_workspace_bytes.restype = ctypes.c_size_t
        lib.mot_workspace_bytes.argtypes = [ctypes.POINTER(_Shapes)]
        lib.mot_depth_ratio_map.restype = ctypes.c_int
        lib.mot_depth_ratio_map.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]
        lib.mot_status_string.restype = ctypes.c_char_p
        lib.mot_status_string.argtypes = [ctypes.c_int]
        lib.mot_last_error.restype = ctypes.c_char_p
        lib.mot_abi_version.restype = ctypes.c_int
        lib.mot_restore_kv.restype = ctypes.c_int
        lib.mot_restore_kv.argtypes = [ctypes.c_void_p] * 8 + [ctypes.POINTER(_RestoreShapes),
                                                               ctypes.c_void_p]
        lib.mot_topS_select.restype = ctypes.c_int
        lib.mot_topS_select.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_ReplayShapes),
                                        ctypes.c_void_p]
        lib.mot_backbone_param_count.restype = ctypes.c_size_t
        lib.mot_backbone_param_count.argtypes = [ctypes.POINTER(_Shapes), ctypes.POINTER(_BackboneDims)]
        lib.mot_backbone_translate.restype = ctypes.c_int
        lib.mot_backbone_translate.argtypes = [ctypes.c_void_p] * 4 + [ctypes.POINTER(_RW), ctypes.c_void_p,
                                                                       ctypes.c_void_p, ctypes.POINTER(_Shapes),
                                                                       ctypes.POINTER(_BackboneDims), ctypes.c_void_p]
        lib.mot_replay_workspace_bytes.restype = ctypes.c_size_t
        lib.mot_replay_workspace_bytes.argtypes = [ctypes.POINTER(_ReplayShapes), ctypes.c_int]
        lib.mot_backbone_workspace_bytes.restype = ctypes.c_size_t
        lib.mot_backbone_workspace_bytes.argtypes = [ctypes.POINTER(_Shapes), ctypes.POINTER(_BackboneDims)]
        lib.mot_usage_stats.restype = ctypes.c_int
        lib.mot_usage_stats.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                        ctypes.c_void_p, ctypes.c_void_p]
        for fn in (lib.mot_replay_attention, lib.mot_replay_attention_noalloc):
            fn.restype = ctypes.c_int
            fn.argtypes = [ctypes.c_void_p] * 5 + [ctypes.POINTER(_ReplayShapes), ctypes.c_void_p]
        P = ctypes.c_void_p
        for name, res, args in (("mot_paged_attention", ctypes.c_int, [P] * 10),
                                ("mot_attend_workspace_bytes", ctypes.c_size_t, [P] * 2),
                                ("mot_cache_append", ctypes.c_int, [P] * 13),
                                ("mot_cache_reorder", ctypes.c_int, [P] * 9 + [ctypes.c_int32, P, ctypes.c_size_t, P]),
                                ("mot_cache_compact", ctypes.c_int, [P] * 7 + [ctypes.c_size_t, P]),
                                ("mot_cache_workspace_bytes", ctypes.c_size_t, [P, ctypes.c_int32])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def abi_version() -> int:
    return load_library().mot_abi_version()


def status_string(status: int) -> str:
    return load_library().mot_status_string(status).decode()


def _check(rc: int):
    if rc != 0:
        raise MotError(rc, load_library().mot_last_error().decode())


def depth_ratio_map(L_src: int, L_tgt: int):
    import numpy as np
    out = np.zeros(L_tgt, dtype=np.int32)
    _check(load_library().mot_depth_ratio_map(L_src, L_tgt, out.ctypes.data))
    return out


def workspace_bytes(shapes: Shapes) -> int:
    c = shapes.c()
    n = load_library().mot_workspace_bytes(ctypes.byref(c))
    if n == ctypes.c_size_t(-1).value:
        raise MotError(2, load_library().mot_last_error().decode())
    return int(n)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def translate_raw(src_k, src_v, layer_map, w1, b1, w2, b2, wr, br, dst_k, dst_v,
                  shapes: Shapes, stream=None, workspace=None, workspace_bytes_=0, usage=None) -> None:
    """Call mot_translate with raw device addresses (ints) or tensors.  No
    checks beyond the library's own (used by the ABI validation tests)."""
    import numpy as np
    lib = load_library()
    lm = np.ascontiguousarray(layer_map, dtype=np.int32)
    tw = _TW(_ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2))
    rw = _RW(_ptr(wr), _ptr(br))
    c = shapes.c(_ptr(workspace), workspace_bytes_, _ptr(usage))
    _check(lib.mot_translate(_ptr(src_k), _ptr(src_v), lm.ctypes.data if lm.size else None,
                             ctypes.byref(tw), ctypes.byref(rw), _ptr(dst_k), _ptr(dst_v),
                             ctypes.byref(c), stream))


def translate_scratch_bytes(shapes: Shapes, layer_map: Sequence[int]) -> int:
    """Bytes of scratch with which ``translate`` splits the last tiles of the
    fused dense path for a call of these shapes; 0 when it would not."""
    import numpy as np
    lm = np.ascontiguousarray(layer_map, dtype=np.int32)
    if lm.size != shapes.L_tgt:
        return 0
    c = shapes.c()
    return int(load_library().mot_translate_scratch_bytes(ctypes.byref(c), lm.ctypes.data))


def _captured_outside_torch(dev) -> bool:
    """Whether the current stream is being captured into a graph that torch's
    allocator does not know of: memory taken from it now would be handed out
    again when the call returns, while the graph goes on writing to it.  (Under
    torch.cuda.graph allocations come from the graph's own pool.)"""
    import torch
    if not torch.cuda.is_current_stream_capturing():
        return False
    probe = torch.empty(1, dtype=torch.uint8, device=dev)
    at = probe.data_ptr()
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= at < seg["address"] + seg["total_size"]:
            return tuple(seg.get("segment_pool_id", (0, 0))) == (0, 0)
    return True


def translate(src_k, src_v, layer_map: Sequence[int], w1, b1, w2, b2, wr, br, dst_k, dst_v,
              shapes: Shapes, workspace=None, usage=None, scratch=None) -> None:
    """Translate on the current torch stream.  Tensors must live on the
    current HIP device, be contiguous and have the dtype named by
    ``shapes.dtype`` (torch.float32 or torch.bfloat16).  ``usage``: optional
    int32 tensor [L_tgt][streams][E] of translator selection counts that the
    call adds to (the library treats it as uint32).

    ``scratch``: memory for the split tiles of the fused dense path
    (mot_translate_scratch).  None: taken from torch's allocator for this call
    where the call splits (none under a capture begun outside torch).  A
    contiguous tensor on the device: used if it holds
    ``translate_scratch_bytes``, and nothing is allocated.  False: no split, so a
    token's row has the same bits whatever other tokens the call holds."""
    import numpy as np
    import torch
    want = torch.float32 if shapes.dtype == MOT_F32 else torch.bfloat16
    dev = torch.device("cuda", torch.cuda.current_device())
    for name, t in (("src_k", src_k), ("src_v", src_v), ("w1", w1), ("b1", b1), ("w2", w2),
                    ("b2", b2), ("wr", wr), ("br", br), ("dst_k", dst_k), ("dst_v", dst_v)):
        if t is None:
            continue
        if t.device != dev:
            raise MotError(1, "%s is on %s, expected %s" % (name, t.device, dev))
        if t.dtype != want:
            raise MotError(2, "%s has dtype %s, expected %s" % (name, t.dtype, want))
        if not t.is_contiguous():
            raise MotError(2, "%s is not contiguous" % name)
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = workspace.numel() * workspace.element_size()
    if usage is not None and (usage.device != dev or usage.dtype != torch.int32 or not usage.is_contiguous()):
        raise MotError(2, "usage must be a contiguous int32 tensor on %s" % dev)
    lib = load_library()
    lm = np.ascontiguousarray(layer_map, dtype=np.int32)
    c = shapes.c(_ptr(workspace), ws_bytes, _ptr(usage))
    n = 0
    if scratch is None:
        # allocated for this call on the current stream, so torch's allocator
        # orders its reuse (under torch.cuda.graph too); without room for it the
        # call runs unsplit
        if shapes.dtype == MOT_BF16 and lm.size == shapes.L_tgt:
            n = lib.mot_translate_scratch_bytes(ctypes.byref(c), lm.ctypes.data)
        if n and _captured_outside_torch(dev):
            n = 0
        if n:
            try:
                scratch = torch.empty(n, dtype=torch.uint8, device=dev)
            except torch.cuda.OutOfMemoryError:
                n = 0
    elif scratch is False:
        scratch = None
    else:
        if scratch.device != dev or not scratch.is_contiguous():
            raise MotError(2, "scratch must be a contiguous tensor on %s" % dev)
        n = scratch.numel() * scratch.element_size()
    tw = _TW(_ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2))
    rw = _RW(_ptr(wr), _ptr(br))
    _check(lib.mot_translate_scratch(_ptr(src_k), _ptr(src_v), lm.ctypes.data if lm.size else None,
                                     ctypes.byref(tw), ctypes.byref(rw), _ptr(dst_k), _ptr(dst_v), ctypes.byref(c),
                                     _ptr(scratch), n, torch.cuda.current_stream().cuda_stream))


def usage_stats(counts, cv2, entropy) -> None:
    """mot_usage_stats on the current torch stream: counts int32 [n][E]
    (read as uint32), cv2 and entropy float64 [n] (outputs)."""
    import torch
    for name, t, dt in (("counts", counts, torch.int32), ("cv2", cv2, torch.float64),
                        ("entropy", entropy, torch.float64)):
        if t.dtype != dt or not t.is_contiguous():
            raise MotError(2, "%s must be a contiguous %s tensor" % (name, dt))
    n, E = counts.shape
    _check(load_library().mot_usage_stats(_ptr(counts), n, E, _ptr(cv2), _ptr(entropy),
                                          torch.cuda.current_stream().cuda_stream))


def restore_kv(act, layer_map, wk, bk, wv, bv, dst_k, dst_v, L: int, B: int, T: int, d_act: int,
               H_tgt: int, D_tgt: int, dst_layout: int = LAYOUT_BTHD) -> None:
    """mot_restore_kv on the current torch stream (bf16 tensors on the
    current device): K = W^K a + b^K and V = W^V a + b^V for every layer with
    layer_map[l] >= 0 (layer_map None = all layers)."""
    import numpy as np
    import torch
    lib = load_library()
    for name, t in (("act", act), ("wk", wk), ("bk", bk), ("wv", wv), ("bv", bv), ("dst_k", dst_k),
                    ("dst_v", dst_v)):
        if t is not None and (t.dtype != torch.bfloat16 or not t.is_contiguous()):
            raise MotError(2, "%s must be a contiguous bfloat16 tensor" % name)
    lm = None if layer_map is None else np.ascontiguousarray(layer_map, dtype=np.int32)
    c = _RestoreShapes(L, B, T, d_act, H_tgt, D_tgt, MOT_BF16, dst_layout)
    stream = torch.cuda.current_stream().cuda_stream
    _check(lib.mot_restore_kv(_ptr(act), lm.ctypes.data if lm is not None else None, _ptr(wk),
                              _ptr(bk), _ptr(wv), _ptr(bv), _ptr(dst_k), _ptr(dst_v),
                              ctypes.byref(c), stream))


def topS_select(A, idx, B: int, T: int, S: int) -> None:
    """mot_topS_select on the current torch stream: A fp32 [B][T][T] (head-
    averaged source attention), idx int32 [B][T][S] (output)."""
    import torch
    lib = load_library()
    for name, t, dt in (("A", A, torch.float32), ("idx", idx, torch.int32)):
        if t is not None and (t.dtype != dt or not t.is_contiguous()):
            raise MotError(2, "%s must be a contiguous %s tensor" % (name, dt))
    c = _ReplayShapes(B, T, 1, 1, 128, S, LAYOUT_BTHD)
    _check(lib.mot_topS_select(_ptr(A), _ptr(idx), ctypes.byref(c),
                               torch.cuda.current_stream().cuda_stream))


def replay_workspace_bytes(B: int, T: int, H_q: int, H_kv: int, D: int, S: int = 0, with_sets: bool = False) -> int:
    c = _ReplayShapes(B, T, H_q, H_kv, D, S, LAYOUT_BTHD)
    n = load_library().mot_replay_workspace_bytes(ctypes.byref(c), int(with_sets))
    if n == ctypes.c_size_t(-1).value:
        raise MotError(2, load_library().mot_last_error().decode())
    return int(n)


def replay_attention(q, k, v, idx, o, B: int, T: int, H_q: int, H_kv: int, D: int, S: int = 0,
                     kv_layout: int = LAYOUT_BTHD, workspace=None) -> None:
    """mot_replay_attention on the current torch stream (bf16 q, k, v, o;
    int32 idx [B][T][S], or None for the full causal set; optional device
    workspace tensor for the full causal set's staging)."""
    import torch
    lib = load_library()
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        if t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise MotError(2, "%s must be a contiguous bfloat16 tensor" % name)
    if idx is not None and (idx.dtype != torch.int32 or not idx.is_contiguous()):
        raise MotError(2, "idx must be a contiguous int32 tensor")
    c = _ReplayShapes(B, T, H_q, H_kv, D, S if idx is not None else 0, kv_layout, _ptr(workspace),
                      workspace.numel() * workspace.element_size() if workspace is not None else 0)
    _check(lib.mot_replay_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(idx), _ptr(o), ctypes.byref(c),
                                    torch.cuda.current_stream().cuda_stream))


def replay_attention_noalloc(q, k, v, idx, o, B: int, T: int, H_q: int, H_kv: int, D: int, S: int = 0,
                             kv_layout: int = LAYOUT_BTHD) -> None:
    """mot_replay_attention_noalloc on the current torch stream: the same
    operation as replay_attention, with the full causal path's staging in the
    library's static per-device scratch (no allocation)."""
    import torch
    lib = load_library()
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        if t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise MotError(2, "%s must be a contiguous bfloat16 tensor" % name)
    if idx is not None and (idx.dtype != torch.int32 or not idx.is_contiguous()):
        raise MotError(2, "idx must be a contiguous int32 tensor")
    c = _ReplayShapes(B, T, H_q, H_kv, D, S if idx is not None else 0, kv_layout)
    _check(lib.mot_replay_attention_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(idx), _ptr(o), ctypes.byref(c),
                                            torch.cuda.current_stream().cuda_stream))


def backbone_param_count(shapes: Shapes, d_h: int, n_heads: int, d_ff: int, n_slots: int = 1) -> int:
    """Elements per expert of the packed backbone parameters."""
    c = shapes.c()
    return int(load_library().mot_backbone_param_count(ctypes.byref(c),
                                                       ctypes.byref(_BackboneDims(d_h, n_heads, d_ff, n_slots))))


def backbone_workspace_bytes(shapes: Shapes, d_h: int, n_heads: int, d_ff: int, n_slots: int = 1) -> int:
    c = shapes.c()
    n = load_library().mot_backbone_workspace_bytes(ctypes.byref(c),
                                                    ctypes.byref(_BackboneDims(d_h, n_heads, d_ff, n_slots)))
    if n == ctypes.c_size_t(-1).value:
        raise MotError(2, load_library().mot_last_error().decode())
    return int(n)


def backbone_translate(src_k, src_v, layer_map, params, wr, br, dst_k, dst_v, shapes: Shapes, d_h: int,
                       n_heads: int, d_ff: int, usage=None, workspace=None, n_slots: int = 1) -> None:
    """mot_backbone_translate on the current torch stream (bf16 tensors)."""
    import numpy as np
    import torch
    lib = load_library()
    for name, t in (("src_k", src_k), ("src_v", src_v), ("params", params), ("wr", wr), ("br", br),
                    ("dst_k", dst_k), ("dst_v", dst_v)):
        if t is not None and (t.dtype != torch.bfloat16 or not t.is_contiguous()):
            raise MotError(2, "%s must be a contiguous bfloat16 tensor" % name)
    lm = np.ascontiguousarray(layer_map, dtype=np.int32)
    rw = _RW(_ptr(wr), _ptr(br))
    c = shapes.c(_ptr(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0,
                 _ptr(usage))
    _check(lib.mot_backbone_translate(_ptr(src_k), _ptr(src_v), lm.ctypes.data, _ptr(params), ctypes.byref(rw),
                                      _ptr(dst_k), _ptr(dst_v), ctypes.byref(c),
                                      ctypes.byref(_BackboneDims(d_h, n_heads, d_ff, n_slots)),
                                      torch.cuda.current_stream().cuda_stream))


# the paged cache --------------------------------------------------------------------------------------------------
#
# A decoding step's kernels take a few microseconds, so these calls keep their own
# share small: sizes go to the library as packed bytes (the layouts of
# _CacheShapes, _AttendShapes, _AppendShapes and _Rope), checks first, texts only
# for what fails them.

_CACHE = struct.Struct("9i")
_ATTEND = struct.Struct("5if8q")
_APPEND = struct.Struct("5if16q")
_ROPE = struct.Struct("4P")
_SCRATCH = struct.Struct("PN")
_NO_STRIDES = (0, 0, 0, 0)
_torch = None


def _ready():
    """(the library, torch), loaded."""
    global _torch
    if _torch is None:
        import torch
        lib, _torch = load_library(), torch
    return _lib, _torch


def _refuse(status: int, detail: str):
    raise MotError(status, detail)


def _stream(dev: int) -> int:
    return _torch._C._cuda_getCurrentRawStream(dev)


class _Pools:
    """The cache's shapes from its tensors: pools [L][n_pages] x page or one
    layer's [n_pages] x page, table int32 [B][max_pages]."""
    __slots__ = ("packed", "dtype", "dev", "L", "heads", "D", "B", "max_pages")

    def __init__(self, k_pages, v_pages, table, page_layout: int):
        torch = _torch
        shape, dtype, dev = k_pages.shape, k_pages.dtype, k_pages.get_device()
        n = len(shape)
        if n not in (4, 5) or shape != v_pages.shape:
            _refuse(2, "k_pages and v_pages must be alike, [L][n_pages] or [n_pages] x a page of three axes")
        code = MOT_BF16 if dtype is torch.bfloat16 else MOT_F32
        if v_pages.dtype is not dtype or (code == MOT_F32 and dtype is not torch.float32):
            _refuse(2, "the pools must be float32 or bfloat16 both, not %s, %s" % (dtype, v_pages.dtype))
        if not (k_pages.is_contiguous() and v_pages.is_contiguous()):
            _refuse(2, "the pools must be contiguous")
        if dev < 0 or v_pages.get_device() != dev or dev != torch._C._cuda_getDevice():
            _refuse(1, "the pools are on %s and %s, expected the current device" % (k_pages.device, v_pages.device))
        self.dev, self.dtype = dev, dtype
        self.ints(table, "table", 2)
        self.B, self.max_pages = table.shape
        self.L = shape[0] if n == 5 else 0      # 0: no axis of layers
        page, self.heads, self.D = shape[-3:]
        if page_layout == LAYOUT_BHTD:
            page, self.heads = self.heads, page
        self.packed = _CACHE.pack(self.L if n == 5 else 1, shape[-4], page, self.heads, self.D, self.B, self.max_pages,
                                  code, page_layout)

    def ints(self, t, name: str, dims: int, n: Optional[int] = None) -> int:
        """Address of an int32 tensor."""
        if t.dtype is not _torch.int32 or t.dim() != dims or not t.is_contiguous() or t.get_device() != self.dev:
            _refuse(2, "%s must be a contiguous int32 tensor of %d axes on the pools' device" % (name, dims))
        if n is not None and t.numel() != n:
            _refuse(2, "%s has %d entries, expected %d" % (name, t.numel(), n))
        return t.data_ptr()

    def rows(self, t, name: str, lead: tuple, heads: int) -> tuple:
        """Strides (layer, batch, token, head) of a row tensor [L] x lead x
        [heads][D] of the pools' type and device."""
        want = ((self.L,) if self.L else ()) + lead + (heads, self.D)
        if t.shape != want:
            _refuse(2, "%s has shape %s, expected %s" % (name, tuple(t.shape), want))
        if t.dtype is not self.dtype or t.get_device() != self.dev:
            _refuse(2, "%s is %s on %s, expected the pools' %s on device %d" % (name, t.dtype, t.device, self.dtype, self.dev))
        st = t.stride()
        if st[-1] != 1 and self.D > 1:
            _refuse(2, "%s has a stride of %d between a head's elements" % (name, st[-1]))
        return (st[0] if self.L else 0, st[-4] if len(lead) == 2 else 0, st[-3], st[-2])

    def new_rows(self, t, name: str, new_start, max_new) -> tuple:
        """(leading axes, n_new, max_new) of a call's row tensor."""
        lead = tuple(t.shape[1 if self.L else 0:-2])
        axes = "[L]" if self.L else ""
        if new_start is None:
            if len(lead) != 2 or lead[0] != self.B:
                _refuse(2, "%s must be %s[B = %d][new tokens][heads][D] without new_start" % (name, axes, self.B))
            if max_new is not None and max_new != lead[1]:
                _refuse(2, "max_new = %d, but %s has %d tokens per sequence" % (max_new, name, lead[1]))
            return lead, lead[0] * lead[1], lead[1]
        if len(lead) != 1:
            _refuse(2, "%s must be %s[new tokens][heads][D] with new_start" % (name, axes))
        return lead, lead[0], lead[0] if max_new is None else min(int(max_new), lead[0])

    def scratch(self, nbytes: int, given, name: str) -> tuple:
        """(tensor or None, address, bytes) of a call's scratch: the given one, or
        torch memory of the current stream."""
        if given is not None:
            if given.get_device() != self.dev or not given.is_contiguous():
                _refuse(2, "%s must be a contiguous tensor on the pools' device" % name)
            return given, given.data_ptr(), given.numel() * given.element_size()
        if not nbytes:
            return None, 0, 0
        dev = _torch.device("cuda", self.dev)
        if _captured_outside_torch(dev):
            return None, 0, 0
        held = _torch.empty(nbytes, dtype=_torch.uint8, device=dev)
        return held, held.data_ptr(), nbytes


def _sized(n: int) -> int:
    if n == _SIZE_MAX:
        raise MotError(2, _lib.mot_last_error().decode())
    return n


def paged_attention(q, k_pages, v_pages, table, kv_len, o, new_start=None, max_new: Optional[int] = None,
                    window: int = 0, scale: Optional[float] = None, max_kv: int = 0, page_layout: int = LAYOUT_BTHD,
                    scratch=None) -> None:
    """mot_paged_attention on the current torch stream: the new tokens' attention
    over one layer's pages, k_pages and v_pages [n_pages][page_size][H_kv][D]
    (LAYOUT_BTHD) or [n_pages][H_kv][page_size][D] (LAYOUT_BHTD).

    q, o: [B][new][H_q][D], or with new_start (int32 [B + 1]) packed
    [tokens][H_q][D]; any strides with contiguous heads.  kv_len int32 [B] counts
    the new tokens, max_new (packed; default: all rows) bounds those of a
    sequence.  window 0: all positions up to the token's.

    ``scratch``: memory for calls that cut long sequences.  None: taken from
    torch's allocator for this call (none under a capture begun outside torch).
    A contiguous tensor: used if it suffices.  False: no cuts."""
    lib, _ = _ready()
    c = _Pools(k_pages, v_pages, table, page_layout)
    if c.L or k_pages.dim() != 4:
        _refuse(2, "attention reads one layer's pools, [n_pages] x page")
    kv = c.ints(kv_len, "kv_len", 1, c.B)
    start = None if new_start is None else c.ints(new_start, "new_start", 1, c.B + 1)
    if q.dim() < 3:
        _refuse(2, "q must be [B][new][H_q][D] or [tokens][H_q][D]")
    lead, n_new, mx = c.new_rows(q, "q", new_start, max_new)
    H_q = q.shape[-2]
    if scale is not None and not 1.2e-38 <= scale <= 3.4e38:
        _refuse(2, "scale must be a positive float32")
    if not (0 <= window < 1 << 31 and 0 <= max_kv < 1 << 31):
        _refuse(2, "window = %s and max_kv = %s must be in [0, 2^31)" % (window, max_kv))
    sizes = _ATTEND.pack(n_new, mx, H_q, window, max_kv, scale or 0.0, *c.rows(q, "q", lead, H_q), *c.rows(o, "o", lead, H_q))
    held, at, nbytes = None, 0, 0
    if scratch is not False:
        need = 0 if scratch is not None else _sized(lib.mot_attend_workspace_bytes(c.packed, sizes + _SCRATCH.pack(0, 0)))
        held, at, nbytes = c.scratch(need, scratch, "scratch")
    rc = lib.mot_paged_attention(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), kv, start,
                                 o.data_ptr(), c.packed, sizes + _SCRATCH.pack(at, nbytes), _stream(c.dev))
    if rc:
        _check(rc)


def cache_append(q, k, v, q_out, k_pages, v_pages, table, kv_len, new_start=None, max_new: Optional[int] = None,
                 q_gain=None, k_gain=None, eps: float = 1e-6, inv_freq=None, interleaved: bool = False,
                 positions=None, page_layout: int = LAYOUT_BTHD) -> None:
    """mot_cache_append on the current torch stream: queries and keys normed per
    head (q_gain, k_gain [D] or [L][D]) and rotated (inv_freq float32
    [rotary_dim / 2]), queries to q_out, keys and values into their pages.

    Pools of one layer [n_pages] x page with rows [B][new][heads][D] (packed with
    new_start: [tokens][heads][D]), or of L layers [L][n_pages] x page with rows
    [L] x those; any strides with contiguous heads.  q and q_out may be None, or
    the same tensor; k and v may be None."""
    lib, torch = _ready()
    c = _Pools(k_pages, v_pages, table, page_layout)
    kv = c.ints(kv_len, "kv_len", 1, c.B)
    start = None if new_start is None else c.ints(new_start, "new_start", 1, c.B + 1)
    some = q if k is None else k
    if some is None or (q is None) != (q_out is None) or (k is None) != (v is None):
        _refuse(1, "q with q_out, k with v, and one pair at least")
    if some.dim() < 3 + (c.L > 0):
        _refuse(2, "rows must be %s[B][new][heads][D] or packed" % ("[L]" if c.L else ""))
    lead, n_new, mx = c.new_rows(some, "q" if k is None else "k", new_start, max_new)
    if not 0 <= eps <= 3.4e38:
        _refuse(2, "eps must be >= 0 and finite")
    H_q = rot = 0
    qs = qos = ks = vs = _NO_STRIDES
    if q is not None:
        H_q = q.shape[-2]
        qs, qos = c.rows(q, "q", lead, H_q), c.rows(q_out, "q_out", lead, H_q)
    if k is not None:
        ks, vs = c.rows(k, "k", lead, c.heads), c.rows(v, "v", lead, c.heads)
    for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
        if g is not None and (g.dtype is not c.dtype or g.get_device() != c.dev or g.numel() != (c.L or 1) * c.D
                              or not g.is_contiguous()):
            _refuse(2, "%s must be contiguous, [L][D], of the pools' type and device" % name)
    if inv_freq is not None:
        if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or inv_freq.get_device() != c.dev:
            _refuse(2, "inv_freq must be a contiguous float32 vector on the pools' device")
        rot = 2 * inv_freq.numel()
        if rot == 0:
            _refuse(2, "inv_freq is empty")
    pos = 0 if positions is None else c.ints(positions, "positions", positions.dim(), n_new)
    rope = _ROPE.pack(0 if q_gain is None else q_gain.data_ptr(), 0 if k_gain is None else k_gain.data_ptr(),
                      0 if inv_freq is None else inv_freq.data_ptr(), pos)
    rc = lib.mot_cache_append(_ptr(q), _ptr(k), _ptr(v), _ptr(q_out), k_pages.data_ptr(), v_pages.data_ptr(),
                              table.data_ptr(), kv, start, rope, c.packed,
                              _APPEND.pack(n_new, mx, H_q, rot, interleaved, eps, *qs, *qos, *ks, *vs), _stream(c.dev))
    if rc:
        _check(rc)


def cache_workspace_bytes(k_pages, v_pages, table, n_rows: int, page_layout: int = LAYOUT_BTHD) -> int:
    """Bytes of workspace of cache_reorder for n_rows new rows (0: of
    cache_compact)."""
    lib, _ = _ready()
    return _sized(lib.mot_cache_workspace_bytes(_Pools(k_pages, v_pages, table, page_layout).packed, n_rows))


def _pages_workspace(c: _Pools, n_rows: int, given) -> tuple:
    need = _sized(_lib.mot_cache_workspace_bytes(c.packed, n_rows))
    held, at, nbytes = c.scratch(need, given, "workspace")
    if held is None and need:
        _refuse(1, "under a capture begun outside torch the call needs a workspace of %d bytes" % need)
    return held, at, nbytes


def cache_reorder(k_pages, v_pages, table, source, keep, want, new_table, missing, page_layout: int = LAYOUT_BTHD,
                  workspace=None) -> None:
    """mot_cache_reorder on the current torch stream: row b of new_table takes the
    first keep[b] positions of row source[b] of table and room for want[b]
    (int32 [n_rows] each; missing: int32 [1], output).  source -1: nothing is
    kept; a row that ends has want 0 too, a new prompt's its length.  workspace None: torch
    memory of this call."""
    lib, _ = _ready()
    c = _Pools(k_pages, v_pages, table, page_layout)
    n = source.numel()
    src, kp, wt = c.ints(source, "source", 1), c.ints(keep, "keep", 1, n), c.ints(want, "want", 1, n)
    new, short = c.ints(new_table, "new_table", 2), c.ints(missing, "missing", 1, 1)
    if new_table.shape != (n, c.max_pages):
        _refuse(2, "new_table has shape %s, expected %s" % (tuple(new_table.shape), (n, c.max_pages)))
    held, at, nbytes = _pages_workspace(c, n, workspace)
    rc = lib.mot_cache_reorder(k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), src, kp, wt, new, short, c.packed,
                               n, at, nbytes, _stream(c.dev))
    if rc:
        _check(rc)


def cache_compact(k_pages, v_pages, table, new_table, used, page_layout: int = LAYOUT_BTHD, workspace=None) -> None:
    """mot_cache_compact on the current torch stream: the pages that table names
    move to the lowest numbers; new_table int32 like table and used int32 [1]
    are outputs.  workspace None: torch memory of this call."""
    lib, _ = _ready()
    c = _Pools(k_pages, v_pages, table, page_layout)
    new, n = c.ints(new_table, "new_table", 2), c.ints(used, "used", 1, 1)
    if new_table.shape != table.shape:
        _refuse(2, "new_table has shape %s, expected %s" % (tuple(new_table.shape), tuple(table.shape)))
    held, at, nbytes = _pages_workspace(c, 0, workspace)
    rc = lib.mot_cache_compact(k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), new, n, c.packed, at, nbytes,
                               _stream(c.dev))
    if rc:
        _check(rc)
