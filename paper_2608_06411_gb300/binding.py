"""Thin ctypes binding of libmap_gb300 (include/map_gb300.h): argument marshalling only.

Every step of the pruning path runs in the CUDA library; this module passes tensor
pointers, sizes and the current CUDA stream through and turns error codes into
exceptions.  Importing it loads the library and raises ImportError if it is missing:
there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import POINTER, c_double, c_float, c_int, c_int32, c_longlong, c_size_t, c_void_p
from itertools import chain

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmap_gb300.so")

MAP_OK, MAP_EINVAL, MAP_ENOMEM, MAP_ECUDA, MAP_ETIMEOUT, MAP_EUNSUPPORTED, MAP_EINTERNAL = 0, -1, -2, -3, -4, -5, -6
K_GEMM_FV1, K_GEMM_FV2, K_GEMM_WK, K_GEMM_TEXT, K_SCORES, K_SELECT, K_GATHER = range(7)
EPI_GELU_BF16, EPI_BIAS_BF16, EPI_F32 = 0, 1, 3

WEIGHT_NAMES = ("wT1", "bT1", "wT2", "bT2", "wQ", "wV1", "bV1", "wV2", "bV2", "wK")


class MapConfig(ctypes.Structure):
    _fields_ = [("D", c_int), ("Dh", c_int), ("dp", c_int), ("rope_theta", c_float), ("rope_on", c_int),
                ("k0_frac", c_float), ("k0_abs", c_int), ("lam", c_float), ("tau", c_float)]


class MapWeights(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in WEIGHT_NAMES]


class MapGrads(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in WEIGHT_NAMES]


class MapCounters(ctypes.Structure):
    _fields_ = [("launches", c_longlong), ("select_rounds", c_longlong), ("gram_rows", c_longlong)]


# Every symbol the header declares, with its ctypes signature.
SIGNATURES = {
    "map_config_default": (c_int, [POINTER(MapConfig)]),
    "map_init": (c_int, [POINTER(MapConfig), POINTER(MapWeights), POINTER(c_void_p)]),
    "map_score": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), c_int, c_int, c_void_p, c_void_p]),
    "map_select": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p]),
    "map_select_noalloc": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p,
                                   c_void_p]),
    "map_gather": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p]),
    "map_qcts": (c_int, [c_void_p, POINTER(c_int32), c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p,
                         c_void_p, c_void_p, c_void_p, c_void_p]),
    "map_assemble": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, POINTER(c_int32), c_int, c_int, c_int, c_int,
                             c_void_p, c_void_p, c_void_p]),
    "map_score_ragged": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), POINTER(c_int32), c_int, c_int,
                                 c_void_p, c_void_p]),
    "map_select_ragged": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), c_int, c_int, c_int, c_void_p,
                                  c_void_p, c_void_p]),
    "map_prune_ragged": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), POINTER(c_int32), c_int, c_int,
                                 c_int, c_void_p, c_void_p, c_void_p, c_void_p]),
    "map_assemble_ragged": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, POINTER(c_int32), POINTER(c_int32),
                                    c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p]),
    "map_assemble_axes": (c_int, [c_void_p] * 7 + [c_int] * 4 + [c_void_p] * 3),
    "map_rope_init": (c_int, [c_int, c_int, c_int, c_int, POINTER(c_double), POINTER(c_int32), c_double,
                              POINTER(c_void_p)]),
    "map_rope_destroy": (None, [c_void_p]),
    # map_heads and map_cache are passed as packed bytes (c_void_p): see _heads and Cache
    "map_qk_rotate": (c_int, [c_void_p, c_int, c_longlong] + [c_void_p] * 8),
    "map_qk_rotate_grad_workspace": (c_size_t, [c_void_p]),
    "map_qk_rotate_grad": (c_int, [c_void_p, c_int, c_longlong] + [c_void_p] * 13),
    "map_cache_extend": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_longlong, c_void_p, c_void_p]),
    "map_qk_rotate_append": (c_int, [c_void_p, c_void_p, c_int, c_longlong] + [c_void_p] * 9),
    "map_cache_fork": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
    "map_cache_free": (c_int, [c_void_p, c_void_p, c_int, c_void_p]),
    "map_cache_attend_workspace": (c_size_t, [c_void_p]),
    "map_cache_attend": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_int, c_float, c_void_p, c_void_p, c_void_p]),
    "map_cache_attend_shared_workspace": (c_size_t, [c_void_p, c_int, c_int, c_int]),
    "map_cache_attend_shared": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p, c_int, c_float, c_void_p,
                                        c_void_p, c_void_p]),
    "map_cache_attend_weigh_workspace": (c_size_t, [c_void_p, c_int, c_int]),
    "map_cache_attend_weigh": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_int, c_float] + [c_void_p] * 4),
    "map_cache_evict_workspace": (c_size_t, [c_void_p, c_int, c_int]),
    "map_cache_evict": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p]),
    "map_cache_status": (c_int, [c_void_p, c_void_p]),
    "map_distill_grad": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), c_void_p, c_int, c_int, c_void_p,
                                 POINTER(MapGrads), c_void_p]),
    "map_prune": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), c_int, c_int, c_int, c_void_p,
                          c_void_p, c_void_p, c_void_p]),
    "map_status": (c_int, [c_void_p, c_void_p]),
    "map_destroy": (None, [c_void_p]),
    "map_strerror": (ctypes.c_char_p, [c_int]),
    "map_get_counters": (c_int, [c_void_p, POINTER(MapCounters)]),
    "map_set_timing": (c_int, [c_void_p, c_int]),
    "map_set_wait_limit": (c_int, [c_void_p, c_longlong]),
    "map_read_timing": (c_int, [c_void_p, c_int, POINTER(c_double), POINTER(c_longlong)]),
    "map_linear": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p]),
    "map_score_debug": (c_int, [c_void_p, c_void_p, c_void_p, POINTER(c_int32), c_int, c_int, c_void_p, c_void_p,
                                c_void_p, c_void_p]),
}


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() (nvcc, sm_103a)")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


class MapError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {lib.map_strerror(code).decode()} ({code})")


def _check(rc: int, where: str) -> None:
    if rc != MAP_OK:
        raise MapError(rc, where)


def _ptr(t) -> c_void_p:
    if t is None:
        return c_void_p(None)
    if isinstance(t, torch.Tensor):
        if not t.is_contiguous():
            raise ValueError("tensors passed to libmap_gb300 must be contiguous")
        return c_void_p(t.data_ptr())
    if isinstance(t, np.ndarray):
        if not t.flags["C_CONTIGUOUS"]:
            raise ValueError("arrays passed to libmap_gb300 must be C-contiguous")
        return c_void_p(t.ctypes.data)
    raise TypeError(f"unsupported buffer type {type(t)}")


def _stream(stream=None) -> c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return c_void_p(s.cuda_stream)


def _lens(lens) -> tuple:
    arr = np.ascontiguousarray(np.asarray(lens, dtype=np.int32))
    return arr, arr.ctypes.data_as(POINTER(c_int32))


def _host_ints(x, rows: int, cols: int, what: str) -> bytes:
    """int32 [rows] or [rows, cols] as bytes, from an array, or a sequence (of sequences) of whole numbers."""
    if isinstance(x, (np.ndarray, torch.Tensor)):
        x = np.asarray(x)
        if x.dtype.kind not in "iu" or x.shape != ((rows,) if cols == 1 else (rows, cols)):
            raise ValueError(f"{what} must be {rows} x {cols} whole numbers")
        x = x.reshape(-1).tolist()
    elif cols > 1:
        if set(map(len, x)) != {cols}:
            raise ValueError(f"{what} must be {rows} x {cols} whole numbers")
        x = list(chain.from_iterable(x))
    if len(x) != rows * cols:
        raise ValueError(f"{what} must be {rows} x {cols} whole numbers")
    try:
        return struct.pack(f"{rows * cols}i", *x)
    except struct.error as e:
        raise ValueError(f"{what} must be {rows} x {cols} whole numbers: {e}") from None


def default_config() -> MapConfig:
    cfg = MapConfig()
    _check(lib.map_config_default(ctypes.byref(cfg)), "map_config_default")
    return cfg


class Context:
    """One library context (weights copied in at construction)."""

    def __init__(self, weights: dict, D: int, Dh: int, dp: int, rope_theta: float = 10000.0, rope_on: bool = True,
                 k0_frac: float = 0.5, k0_abs: int = -1, lam: float = 1.0, tau: float = 1e-5):
        self.cfg = MapConfig(D, Dh, dp, rope_theta, int(bool(rope_on)), k0_frac, k0_abs, lam, tau)
        keep = [np.ascontiguousarray(weights[n]) if isinstance(weights[n], np.ndarray) else weights[n].contiguous()
                for n in WEIGHT_NAMES]
        w = MapWeights(*[_ptr(t) for t in keep])
        h = c_void_p()
        _check(lib.map_init(ctypes.byref(self.cfg), ctypes.byref(w), ctypes.byref(h)), "map_init")
        self.h = h

    def close(self) -> None:
        if self.h:
            lib.map_destroy(self.h)
            self.h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the path -----------------------------------------------------------------------
    def score(self, text, vis, lens, scores=None, stream=None):
        B, N = vis.shape[0], vis.shape[1]
        if scores is None:
            scores = torch.empty((B, N), dtype=torch.float32, device=vis.device)
        arr, lp = _lens(lens)
        _check(lib.map_score(self.h, _ptr(text), _ptr(vis), lp, B, N, _ptr(scores), _stream(stream)), "map_score")
        return scores

    def score_debug(self, text, vis, lens, stream=None):
        B, N = vis.shape[0], vis.shape[1]
        arr, lp = _lens(lens)
        scores = torch.empty((B, N), dtype=torch.float32, device=vis.device)
        q = torch.empty((int(arr.sum()), self.cfg.dp), dtype=torch.float32, device=vis.device)
        k = torch.empty((B * N, self.cfg.dp), dtype=torch.float32, device=vis.device)
        _check(lib.map_score_debug(self.h, _ptr(text), _ptr(vis), lp, B, N, _ptr(scores), _ptr(q), _ptr(k),
                                   _stream(stream)), "map_score_debug")
        return scores, q, k

    def select(self, scores, vis, k: int, keep=None, order=None, want_order: bool = True, stream=None):
        B, N = vis.shape[0], vis.shape[1]
        if keep is None:
            keep = torch.empty((B, k), dtype=torch.int32, device=vis.device)
        if order is None and want_order:
            order = torch.empty((B, k), dtype=torch.int32, device=vis.device)
        _check(lib.map_select(self.h, _ptr(scores), _ptr(vis), B, N, k, _ptr(keep), _ptr(order), _stream(stream)),
               "map_select")
        return keep, order

    def select_noalloc(self, scores, vis, k: int, keep, order=None, stream=None):
        """map_select_noalloc: the caller provides keep (and order) buffers; nothing is
        allocated during the call."""
        B, N = vis.shape[0], vis.shape[1]
        _check(lib.map_select_noalloc(self.h, _ptr(scores), _ptr(vis), B, N, k, _ptr(keep), _ptr(order),
                                      _stream(stream)), "map_select_noalloc")
        return keep, order

    def gather(self, vis, keep, out=None, stream=None):
        B, N, D = vis.shape
        k = keep.shape[1]
        if out is None:
            out = torch.empty((B, k, D), dtype=vis.dtype, device=vis.device)
        _check(lib.map_gather(self.h, _ptr(vis), _ptr(keep), B, N, k, _ptr(out), _stream(stream)), "map_gather")
        return out

    def assemble(self, vis, keep, text, lens, pos_offset: int = 0, seq=None, pos=None, stream=None):
        """map_assemble: per image, the kept tokens then the question tokens, with position ids."""
        B, N, D = vis.shape
        k = keep.shape[1]
        arr, lp = _lens(lens)
        rows = B * k + int(arr.sum())
        if seq is None:
            seq = torch.empty((rows, D), dtype=vis.dtype, device=vis.device)
        if pos is None:
            pos = torch.empty(rows, dtype=torch.int32, device=vis.device)
        _check(lib.map_assemble(self.h, _ptr(vis), _ptr(keep), _ptr(text), lp, B, N, k, pos_offset, _ptr(seq),
                                _ptr(pos), _stream(stream)), "map_assemble")
        return seq, pos

    def assemble_axes(self, vis, keep, text, lens, grids, t_step=None, pos_offset: int = 0, seq=None, pos=None,
                      stream=None):
        """map_assemble_axes: the hand-off sequence with position ids [3, rows] (time, height, width) of images
        that are grids of grids[b] = (T, H, W) tokens, t_step[b] positions from frame to frame (default 1)."""
        B, N, D = vis.shape
        k = keep.shape[1]
        dev, dt = vis.device, vis.dtype
        if dev.type != "cuda" or D != self.cfg.D or vis.element_size() != 2:
            raise ValueError(f"vis must be [B, N, {self.cfg.D}] of a 2-byte type on a CUDA device")
        if stream is not None:               # outputs are allocated on the stream that writes them
            with _on(dev, stream, vis, keep, text, seq, pos):
                return self.assemble_axes(vis, keep, text, lens, grids, t_step, pos_offset, seq, pos)
        m = _host_ints(lens, B, 1, "lens")
        g = _host_ints(grids, B, 3, "grids")
        t = None if t_step is None else _host_ints(t_step, B, 1, "t_step")
        questions = int(sum(lens))
        rows = B * k + questions
        if text.shape[0] < questions or text.shape[1] != D:
            raise ValueError(f"text must be [sum(lens), {D}]")
        if seq is None:
            seq = torch.empty((rows, D), dtype=dt, device=dev)
        if pos is None:
            pos = torch.empty((3, rows), dtype=torch.int32, device=dev)
        _check(lib.map_assemble_axes(self.h, _dense(vis, dt, dev, None, "vis"), _dense(keep, torch.int32, dev, (B, k), "keep"),
                                     _dense(text, dt, dev, None, "text"), m, g, t, B, N, k, pos_offset,
                                     _dense(seq, dt, dev, (rows, D), "seq"), _dense(pos, torch.int32, dev, (3, rows), "pos"),
                                     _current_stream(dev.index)), "map_assemble_axes")
        return seq, pos

    # -- ragged batches (padded layout, n_valid tokens per image) ---------------------------
    def score_ragged(self, text, vis, lens, n_valid, scores=None, stream=None):
        B, N = vis.shape[0], vis.shape[1]
        if scores is None:
            scores = torch.empty((B, N), dtype=torch.float32, device=vis.device)
        arr, lp = _lens(lens)
        nva, nvp = _lens(n_valid)
        _check(lib.map_score_ragged(self.h, _ptr(text), _ptr(vis), lp, nvp, B, N, _ptr(scores), _stream(stream)),
               "map_score_ragged")
        return scores

    def select_ragged(self, scores, vis, n_valid, k: int, keep=None, order=None, want_order: bool = True,
                      stream=None):
        B, N = vis.shape[0], vis.shape[1]
        if keep is None:
            keep = torch.empty((B, k), dtype=torch.int32, device=vis.device)
        if order is None and want_order:
            order = torch.empty((B, k), dtype=torch.int32, device=vis.device)
        nva, nvp = _lens(n_valid)
        _check(lib.map_select_ragged(self.h, _ptr(scores), _ptr(vis), nvp, B, N, k, _ptr(keep), _ptr(order),
                                     _stream(stream)), "map_select_ragged")
        return keep, order

    def prune_ragged(self, text, vis, lens, n_valid, k: int, out, keep, scores=None, stream=None):
        B, N = vis.shape[0], vis.shape[1]
        arr, lp = _lens(lens)
        nva, nvp = _lens(n_valid)
        _check(lib.map_prune_ragged(self.h, _ptr(text), _ptr(vis), lp, nvp, B, N, k, _ptr(out), _ptr(keep),
                                    _ptr(scores), _stream(stream)), "map_prune_ragged")
        return out, keep

    def assemble_ragged(self, vis, keep, text, lens, n_valid, pos_offset: int = 0, seq=None, pos=None,
                        stream=None):
        B, N, D = vis.shape
        k = keep.shape[1]
        arr, lp = _lens(lens)
        nva, nvp = _lens(n_valid)
        rows = B * k + int(arr.sum())
        if seq is None:
            seq = torch.empty((rows, D), dtype=vis.dtype, device=vis.device)
        if pos is None:
            pos = torch.empty(rows, dtype=torch.int32, device=vis.device)
        _check(lib.map_assemble_ragged(self.h, _ptr(vis), _ptr(keep), _ptr(text), lp, nvp, B, N, k, pos_offset,
                                       _ptr(seq), _ptr(pos), _stream(stream)), "map_assemble_ragged")
        return seq, pos

    def distill_grad(self, text, vis, lens, teacher, grads=None, loss=None, stream=None):
        """map_distill_grad: (loss [1], {weight name: fp32 gradient}) on device tensors."""
        B, N = vis.shape[0], vis.shape[1]
        D, Dh, dp = self.cfg.D, self.cfg.Dh, self.cfg.dp
        shapes = {"wT1": (Dh, D), "bT1": (Dh,), "wT2": (Dh, Dh), "bT2": (Dh,), "wQ": (dp, Dh),
                  "wV1": (Dh, D), "bV1": (Dh,), "wV2": (Dh, Dh), "bV2": (Dh,), "wK": (dp, Dh)}
        if grads is None:
            grads = {n: torch.empty(shapes[n], dtype=torch.float32, device=vis.device) for n in WEIGHT_NAMES}
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=vis.device)
        g = MapGrads(*[_ptr(grads[n]) for n in WEIGHT_NAMES])
        arr, lp = _lens(lens)
        _check(lib.map_distill_grad(self.h, _ptr(text), _ptr(vis), lp, _ptr(teacher), B, N, _ptr(loss),
                                    ctypes.byref(g), _stream(stream)), "map_distill_grad")
        return loss, grads

    def prune(self, text, vis, lens, k: int, out, keep, scores=None, stream=None):
        """score + select + gather in one C call; buffers may be host (pinned or not) or device."""
        B, N = vis.shape[0], vis.shape[1]
        arr, lp = _lens(lens)
        _check(lib.map_prune(self.h, _ptr(text), _ptr(vis), lp, B, N, k, _ptr(out), _ptr(keep), _ptr(scores),
                             _stream(stream)), "map_prune")
        return out, keep

    # -- diagnostics and instrumentation -------------------------------------------------
    def linear(self, x, w, b, epi: int, out=None, stream=None):
        M, K = x.shape
        Nout = w.shape[0]
        if out is None:
            dt = torch.float32 if epi == EPI_F32 else torch.bfloat16
            out = torch.empty((M, Nout), dtype=dt, device=x.device)
        _check(lib.map_linear(self.h, _ptr(x), _ptr(w), _ptr(b), M, K, Nout, epi, _ptr(out), _stream(stream)),
               "map_linear")
        return out

    def status(self, stream=None) -> int:
        return lib.map_status(self.h, _stream(stream))

    def check(self, stream=None) -> None:
        _check(self.status(stream), "map_status")

    def counters(self) -> dict:
        c = MapCounters()
        _check(lib.map_get_counters(self.h, ctypes.byref(c)), "map_get_counters")
        return {"launches": c.launches, "select_rounds": c.select_rounds, "gram_rows": c.gram_rows}

    def set_wait_limit(self, ns: int) -> None:
        """Limit of the GEMM kernels' waits in ns (<= 0: the 2 s default); for tests."""
        _check(lib.map_set_wait_limit(self.h, int(ns)), "map_set_wait_limit")

    def set_timing(self, enable: bool) -> None:
        _check(lib.map_set_timing(self.h, int(bool(enable))), "map_set_timing")

    def read_timing(self, kid: int) -> tuple:
        ms, n = c_double(), c_longlong()
        _check(lib.map_read_timing(self.h, kid, ctypes.byref(ms), ctypes.byref(n)), "map_read_timing")
        return ms.value, n.value


def qcts(attn, lens, attn_ref, L: int, H: int, N: int, p=None, p_ref=None, js=None, teacher=None,
         teacher_p=None, want_teacher_p: bool = True, stream=None):
    """map_qcts: Question Contrastive Teacher Selection on device tensors.

    attn: packed bf16 (int16 storage) attention of the B samples ([L, H, lens[b], N] blocks
    in sample order); attn_ref: [B, L, H, M_ref, N].  Returns (p, p_ref, js, teacher,
    teacher_p); outputs not given are allocated here."""
    arr, lp = _lens(lens)
    B = int(arr.shape[0])
    M_ref = int(attn_ref.shape[3])
    dev = attn_ref.device
    if p is None:
        p = torch.empty((B, L, N), dtype=torch.float32, device=dev)
    if p_ref is None:
        p_ref = torch.empty((B, L, N), dtype=torch.float32, device=dev)
    if js is None:
        js = torch.empty((B, L), dtype=torch.float32, device=dev)
    if teacher is None:
        teacher = torch.empty(B, dtype=torch.int32, device=dev)
    if teacher_p is None and want_teacher_p:
        teacher_p = torch.empty((B, N), dtype=torch.float32, device=dev)
    _check(lib.map_qcts(_ptr(attn), lp, _ptr(attn_ref), M_ref, B, L, H, N, _ptr(p), _ptr(p_ref), _ptr(js),
                        _ptr(teacher), _ptr(teacher_p), _stream(stream)), "map_qcts")
    return p, p_ref, js, teacher, teacher_p


# ------------------------------------------------------------------ queries, keys and a cache's pages
# These calls run on the device of the tensors they are given, whichever is current, and on that device's current
# stream unless `stream` is given; scratch and outputs that are not given are allocated on the stream that uses them.
# With `stream` given, inputs have to be ready there (an event, or wait_stream), and may be dropped once the call has returned.
# Autograd does not see these calls: their outputs require no gradient, whatever the inputs do (Rope.grad is rotate's).

TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}      # MAP_BF16, MAP_F16, MAP_F32
CACHE_STATUS_WORDS = 1024                                            # MAP_CACHE_STATUS_WORDS
_pack_heads = struct.Struct("@Pqqi4x").pack                          # map_heads
_pack_cache = struct.Struct("@5P8i").pack                            # map_cache


_current_device = torch._C._cuda_getDevice              # as torch.cuda.current_device and current_stream, without their
_current_stream = torch._C._cuda_getCurrentRawStream    # Python objects: 1.5 us a call less
_capturing = torch._C._cuda_isCurrentStreamCapturing
_KEEP = 1 << 26                                         # bytes of scratch that a Cache keeps


class _on:
    """A device made current, and with a stream of the caller's that one for torch's allocations too.  `tensors` (any of them
    may be None) are what the call reads and writes there: the allocator hears of it, so that the memory of one that the
    caller drops before the stream is done is not handed out before that."""

    def __init__(self, device, stream, *tensors):
        if device.type != "cuda":
            raise ValueError("tensors passed to libmap_gb300 must be on a CUDA device")
        if stream is not None:
            if stream.device != device:
                raise ValueError("the stream is not on the tensors' device")
            for t in tensors:
                if t is not None and t.device == device:        # (others are refused by the call)
                    t.record_stream(stream)
        self.guard = torch.cuda.stream(stream) if stream is not None else torch.cuda.device(device)

    def __enter__(self):
        return self.guard.__enter__()

    def __exit__(self, *exc):
        return self.guard.__exit__(*exc)


def _type(dtype) -> int:
    t = TYPES.get(dtype)
    if t is None:
        raise ValueError(f"unsupported element type {dtype}")
    return t


def _heads(t, rows: int, dh: int, dtype, device):
    """map_heads of a [rows, heads, dh] tensor with any strides but dh's."""
    n, h, d = t.shape
    if n != rows or d != dh or t.dtype is not dtype or t.device != device:
        raise ValueError(f"heads must be [{rows}, heads, {dh}] {dtype} on {device}: got {tuple(t.shape)} {t.dtype} on {t.device}")
    sr, sh, sd = t.stride()
    if sd != 1 and d > 1:
        raise ValueError("a head's columns must be adjacent in memory")
    return _pack_heads(t.data_ptr(), sr, sh, h)


def _like(t, dh: int):
    """A new contiguous tensor of t's shape and type, and its map_heads."""
    out = torch.empty(t.shape, dtype=t.dtype, device=t.device)
    h = t.shape[1]
    return out, _pack_heads(out.data_ptr(), h * dh, dh, h)


def _dense(t, dtype, device, shape=None, what="tensor"):
    """Pointer of a contiguous tensor of the wanted type, place and shape (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor on {device}" + (f" of shape {shape}" if shape else ""))
    return t.data_ptr()


class Rope:
    """A rotation plan (map_rope_init): heads of dh columns, their first 2 * len(inv_freq) rotated; pair i is turned by
    pos[axis[i]] * inv_freq[i].  Serves any stream and device."""

    def __init__(self, dh: int, inv_freq, axis=None, n_axes: int | None = None, adjacent: bool = False, eps: float = 1e-6):
        f = np.ascontiguousarray(np.asarray(inv_freq, dtype=np.float64).reshape(-1))
        a = np.zeros(f.shape[0], np.int32) if axis is None else np.ascontiguousarray(np.asarray(axis, dtype=np.int32).reshape(-1))
        if a.shape != f.shape:
            raise ValueError("axis has one entry a pair")
        self.dh, self.rot = int(dh), 2 * f.shape[0]
        self.n_axes = int(n_axes) if n_axes is not None else (int(a.max()) + 1 if a.size else 1)
        h = c_void_p()
        _check(lib.map_rope_init(self.dh, self.rot, int(bool(adjacent)), self.n_axes, f.ctypes.data_as(POINTER(c_double)),
                                 a.ctypes.data_as(POINTER(c_int32)), float(eps), ctypes.byref(h)), "map_rope_init")
        self.h = h
        self._grad_ws = int(lib.map_qk_rotate_grad_workspace(h))

    def close(self) -> None:
        if self.h:
            lib.map_rope_destroy(self.h)
            self.h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def rotate(self, q, k, pos, wq=None, wk=None, q_out=None, k_out=None, stream=None):
        """map_qk_rotate: (q_out, k_out) of q [rows, heads, dh] and k (either may be None), pos int32 [n_axes, rows],
        norm weights wq, wk [dh] or None (no norm of that side).  Outputs not given are new, contiguous tensors.  Not recorded
        by autograd: a torch.autograd.Function around rotate and grad carries gradients."""
        x = q if q is not None else k
        if x is None:
            raise ValueError("q or k is needed")
        dev = x.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, q, k, pos, wq, wk, q_out, k_out):
                return self.rotate(q, k, pos, wq, wk, q_out, k_out)
        dt, dh, rows = x.dtype, self.dh, x.shape[0]
        a = b = oa = ob = None
        if q is not None:
            a = _heads(q, rows, dh, dt, dev)
            if q_out is None:
                q_out, oa = _like(q, dh)
            else:
                oa = _heads(q_out, rows, dh, dt, dev)
        if k is not None:
            b = _heads(k, rows, dh, dt, dev)
            if k_out is None:
                k_out, ob = _like(k, dh)
            else:
                ob = _heads(k_out, rows, dh, dt, dev)
        _check(lib.map_qk_rotate(self.h, _type(dt), rows, _dense(pos, torch.int32, dev, (self.n_axes, rows), "pos"), a, b,
                                 _dense(wq, dt, dev, (dh,), "wq"), _dense(wk, dt, dev, (dh,), "wk"), oa, ob,
                                 _current_stream(dev.index)), "map_qk_rotate")
        return q_out, k_out

    def grad(self, dq_out, dk_out, pos, q=None, k=None, wq=None, wk=None, dq=None, dk=None, dwq=None, dwk=None,
             stream=None):
        """map_qk_rotate_grad: (dq, dk, dwq, dwk) from the gradients of rotate's outputs; q and k (rotate's inputs) are
        needed where wq and wk are given, dwq and dwk are float32 (None without a norm)."""
        x = dq_out if dq_out is not None else dk_out
        if x is None:
            raise ValueError("dq_out or dk_out is needed")
        dev = x.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, dq_out, dk_out, pos, q, k, wq, wk, dq, dk, dwq, dwk):
                return self.grad(dq_out, dk_out, pos, q, k, wq, wk, dq, dk, dwq, dwk)
        dt, dh, rows, f32 = x.dtype, self.dh, x.shape[0], torch.float32
        a = b = xa = xb = oa = ob = ws = None
        if dq_out is not None:
            a = _heads(dq_out, rows, dh, dt, dev)
            if dq is None:
                dq, oa = _like(dq_out, dh)
            else:
                oa = _heads(dq, rows, dh, dt, dev)
            if wq is not None:
                if q is None:
                    raise ValueError("q is needed with wq")
                xa = _heads(q, rows, dh, dt, dev)
                if dwq is None:
                    dwq = torch.empty(dh, dtype=f32, device=dev)
        if dk_out is not None:
            b = _heads(dk_out, rows, dh, dt, dev)
            if dk is None:
                dk, ob = _like(dk_out, dh)
            else:
                ob = _heads(dk, rows, dh, dt, dev)
            if wk is not None:
                if k is None:
                    raise ValueError("k is needed with wk")
                xb = _heads(k, rows, dh, dt, dev)
                if dwk is None:
                    dwk = torch.empty(dh, dtype=f32, device=dev)
        if xa is not None or xb is not None:
            ws = torch.empty(self._grad_ws, dtype=torch.uint8, device=dev)
        _check(lib.map_qk_rotate_grad(self.h, _type(dt), rows, _dense(pos, torch.int32, dev, (self.n_axes, rows), "pos"), a, b,
                                      xa, xb, _dense(wq, dt, dev, (dh,), "wq"), _dense(wk, dt, dev, (dh,), "wk"), oa, ob,
                                      _dense(dwq, f32, dev, (dh,), "dwq"), _dense(dwk, f32, dev, (dh,), "dwk"),
                                      None if ws is None else ws.data_ptr(), _current_stream(dev.index)), "map_qk_rotate_grad")
        return dq, dk, dwq, dwk

    def append(self, q, k, v, pos, cache, layer: int, slots, wq=None, wk=None, q_out=None, stream=None):
        """map_qk_rotate_append: rotated k, and v, into the cache's slots (Cache.extend); returns the rotated q (None
        without q)."""
        dev = k.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, q, k, v, pos, slots, wq, wk, q_out):
                return self.append(q, k, v, pos, cache, layer, slots, wq, wk, q_out)
        dt, dh, rows = k.dtype, self.dh, k.shape[0]
        if dt != cache.pool.dtype or dev != cache.pool.device:
            raise ValueError("k has the cache's type and device")
        a = oa = None
        if q is not None:
            a = _heads(q, rows, dh, dt, dev)
            if q_out is None:
                q_out, oa = _like(q, dh)
            else:
                oa = _heads(q_out, rows, dh, dt, dev)
        _check(lib.map_qk_rotate_append(self.h, cache.desc, layer, rows, _dense(pos, torch.int32, dev, (self.n_axes, rows), "pos"),
                                        _dense(slots, torch.int32, dev, (rows,), "slots"), a, _heads(k, rows, dh, dt, dev),
                                        _heads(v, rows, dh, dt, dev), _dense(wq, dt, dev, (dh,), "wq"),
                                        _dense(wk, dt, dev, (dh,), "wk"), oa, cache._stream()), "map_qk_rotate_append")
        return q_out


class Cache:
    """Pages of a key/value cache (map_cache) over the caller's tensors: pool [layers, 2, pages, heads, page, dh] bf16 or
    fp16, table int32 [seqs, max_pages], length int32 [seqs], refs int32 [pages], status int32 [CACHE_STATUS_WORDS], the last
    four initially zero (`Cache.empty` makes all of them).  Calls on one cache, replays of captured ones included, are
    ordered by the caller; a graph that holds such calls needs the Cache as long as it is replayed."""

    def __init__(self, pool, table, length, refs, status=None):
        dev = pool.device
        if pool.dim() != 6 or pool.shape[1] != 2 or pool.dtype not in TYPES or not pool.is_contiguous():
            raise ValueError("pool must be a contiguous [layers, 2, pages, heads, page, dh] tensor")
        if status is None:
            status = torch.zeros(CACHE_STATUS_WORDS, dtype=torch.int32, device=dev)
        layers, _, pages, heads, page, dh = pool.shape
        if table.dim() != 2:
            raise ValueError("table must be [seqs, max_pages]")
        seqs, max_pages = table.shape
        ptrs = (_dense(table, torch.int32, dev, None, "table"), _dense(length, torch.int32, dev, (seqs,), "length"),
                _dense(refs, torch.int32, dev, (pages,), "refs"), _dense(status, torch.int32, dev, (CACHE_STATUS_WORDS,), "status"))
        self.pool, self.table, self.length, self.refs, self.status_word = pool, table, length, refs, status
        self.device, self.heads, self.page, self.dh = dev, heads, page, dh
        self._weights_shape = (layers, seqs, heads, max_pages * page)
        self.desc = _pack_cache(pool.data_ptr(), *ptrs, TYPES[pool.dtype], layers, pages, heads, page, dh, seqs, max_pages)
        # attend's scratch: calls on one cache are ordered by the caller, so they can share it
        self._ws = torch.empty(int(lib.map_cache_attend_workspace(self.desc)), dtype=torch.uint8, device=dev)
        self._streams = set()                # that the allocator knows of
        # the other calls', as large as the largest so far (see _scratch)
        self._kept, self._sizes = torch.empty(256, dtype=torch.uint8, device=dev), {}
        self._tensors = (pool, table, length, refs, status, self._ws, self._kept)

    def _stream(self) -> int:
        """The current stream.  The allocator hears of it once, so that the memory of a Cache that is dropped waits for it."""
        st = _current_stream(self.device.index)
        if st not in self._streams:
            for t in self._tensors:
                t.record_stream(torch.cuda.current_stream(self.device))
            self._streams.add(st)
        return st

    @classmethod
    def empty(cls, layers: int, pages: int, heads: int, page: int, dh: int, seqs: int, max_pages: int,
              dtype=torch.bfloat16, device="cuda"):
        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)
        return cls(torch.empty((layers, 2, pages, heads, page, dh), dtype=dtype, device=device), ints(seqs, max_pages),
                   ints(seqs), ints(pages))

    def extend(self, seqs, counts=None, rows: int | None = None, slots=None, stream=None):
        """map_cache_extend: slots int32 [rows] for counts[i] new rows of each sequence seqs[i] (device int32), or with
        counts None for one row each, entry i's at i.  `rows` (or the size of `slots`) is at least their sum and must
        be given with counts."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, seqs, counts, slots):
                return self.extend(seqs, counts, rows, slots)
        n = seqs.shape[0]
        if rows is None:
            if slots is not None:
                rows = slots.shape[0]
            elif counts is None:
                rows = n
            else:
                raise ValueError("rows must be given with counts")
        if slots is None:
            slots = torch.empty(rows, dtype=torch.int32, device=dev)
        _check(lib.map_cache_extend(self.desc, _dense(seqs, torch.int32, dev, (n,), "seqs"),
                                    _dense(counts, torch.int32, dev, (n,), "counts"), n, rows,
                                    _dense(slots, torch.int32, dev, (rows,), "slots"), self._stream()),
               "map_cache_extend")
        return slots

    def fork(self, parents, children, keep=None, base=None, span=None, stream=None) -> None:
        """map_cache_fork: children[i] (empty) gets parents[i]'s rows, with keep int32 [n, k] those of rows
        base[i] .. base[i] + span[i] that keep[i] names (all int32 on the device)."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, parents, children, keep, base, span):
                return self.fork(parents, children, keep, base, span)
        n, i32 = parents.shape[0], torch.int32
        if (keep is None) != (base is None) or (base is None) != (span is None) or (keep is not None and keep.dim() != 2):
            raise ValueError("keep is [n, k] and comes with base and span")
        k = 0 if keep is None else keep.shape[1]
        _check(lib.map_cache_fork(self.desc, _dense(parents, i32, dev, (n,), "parents"),
                                  _dense(children, i32, dev, (n,), "children"), n, _dense(keep, i32, dev, (n, k), "keep"), k,
                                  _dense(base, i32, dev, (n,), "base"), _dense(span, i32, dev, (n,), "span"),
                                  self._stream()), "map_cache_fork")

    def free(self, seqs, stream=None) -> None:
        """map_cache_free: the pages of seqs (int32 [n] on the device) lose a holder, the lengths become 0."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, seqs):
                return self.free(seqs)
        n = seqs.shape[0]
        _check(lib.map_cache_free(self.desc, _dense(seqs, torch.int32, dev, (n,), "seqs"), n, self._stream()),
               "map_cache_free")

    def attend(self, q, seqs, layer: int, scale: float | None = None, out=None, stream=None):
        """map_cache_attend: attention of q [n, heads, dh], row i over all rows of sequence seqs[i] (int32 on the device);
        scale defaults to dh ** -0.5.  Forward only, and without a causal mask: single tokens."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, q, seqs, out):
                return self.attend(q, seqs, layer, scale, out)
        dt, n, dh = self.pool.dtype, seqs.shape[0], self.dh
        a = _heads(q, n, dh, dt, dev)
        if out is None:
            out, oa = _like(q, dh)
        else:
            oa = _heads(out, n, dh, dt, dev)
        _check(lib.map_cache_attend(self.desc, layer, a, _dense(seqs, torch.int32, dev, (n,), "seqs"), n,
                                    dh ** -0.5 if scale is None else scale, oa, self._ws.data_ptr(), self._stream()),
               "map_cache_attend")
        return out

    def _scratch(self, call: str, *args) -> torch.Tensor:
        """A workspace of <call>_workspace(description, *args) bytes.  Up to _KEEP bytes the Cache keeps it for its next calls; a
        larger one is a call's own, and so is one of a call that is captured, whose memory then belongs to the graph."""
        size = self._sizes.get((call, args))
        if size is None:
            if len(self._sizes) >= 4096:     # (calls of ever other sizes)
                self._sizes.clear()
            size = self._sizes[call, args] = int(getattr(lib, call + "_workspace")(self.desc, *args))
        if size > _KEEP or _capturing():
            return torch.empty(max(size, 256), dtype=torch.uint8, device=self.device)
        if size > self._kept.shape[0]:
            self._kept = torch.empty(size, dtype=torch.uint8, device=self.device)
            self._tensors = self._tensors[:-1] + (self._kept,)
            self._streams.clear()            # (the allocator is to hear of it for every stream)
        return self._kept

    def attend_shared(self, q, seqs, layer: int, starts, scale: float | None = None, out=None, stream=None):
        """map_cache_attend_shared: attend, for groups of entries starts[g] .. starts[g + 1] - 1 (int32 [groups + 1] on the
        device, from 0 to n) whose sequences begin with the same pages: those rows are read once for a group."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, q, seqs, starts, out):
                return self.attend_shared(q, seqs, layer, starts, scale, out)
        dt, n, dh, groups = self.pool.dtype, seqs.shape[0], self.dh, starts.shape[0] - 1
        a = _heads(q, n, dh, dt, dev)
        if out is None:
            out, oa = _like(q, dh)
        else:
            oa = _heads(out, n, dh, dt, dev)
        ws = self._scratch("map_cache_attend_shared", q.shape[1], n, groups)
        _check(lib.map_cache_attend_shared(self.desc, layer, a, _dense(seqs, torch.int32, dev, (n,), "seqs"), n,
                                           _dense(starts, torch.int32, dev, (groups + 1,), "starts"), groups,
                                           dh ** -0.5 if scale is None else scale, oa, ws.data_ptr(), self._stream()),
               "map_cache_attend_shared")
        return out

    def attend_weigh(self, q, seqs, layer: int, weights, scale: float | None = None, out=None, stream=None):
        """map_cache_attend_weigh: attend, and each row's attention weight, summed over a key head's query heads, is added to
        weights float32 [layers, seqs, heads, max_pages * page].  Zero a sequence's weights when it begins or is freed."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, q, seqs, weights, out):
                return self.attend_weigh(q, seqs, layer, weights, scale, out)
        dt, n, dh = self.pool.dtype, seqs.shape[0], self.dh
        a = _heads(q, n, dh, dt, dev)
        if out is None:
            out, oa = _like(q, dh)
        else:
            oa = _heads(out, n, dh, dt, dev)
        ws = self._scratch("map_cache_attend_weigh", q.shape[1], n)
        _check(lib.map_cache_attend_weigh(self.desc, layer, a, _dense(seqs, torch.int32, dev, (n,), "seqs"), n,
                                          dh ** -0.5 if scale is None else scale, oa,
                                          _dense(weights, torch.float32, dev, self._weights_shape, "weights"), ws.data_ptr(),
                                          self._stream()), "map_cache_attend_weigh")
        return out

    def evict(self, weights, seqs, first, last, k: int, stream=None) -> None:
        """map_cache_evict: of rows first[i] .. length - last[i] - 1 of sequence seqs[i] the k with the greatest weights stay,
        for each layer and head by itself; the rows behind move up, their weights with them (all int32 on the device, first
        and last None for 0).  Keys stay rotated by the positions they were appended with: count the next token's position
        from the tokens so far, not from `length`."""
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream, weights, seqs, first, last):
                return self.evict(weights, seqs, first, last, k)
        if k >= 1 << 31:                     # (a C int would be what is left of it, and fewer rows stay)
            raise ValueError("k must be below 2^31")
        n, i32 = seqs.shape[0], torch.int32
        ws = self._scratch("map_cache_evict", n, k)
        _check(lib.map_cache_evict(self.desc, _dense(weights, torch.float32, dev, self._weights_shape, "weights"),
                                   _dense(seqs, i32, dev, (n,), "seqs"), n, _dense(first, i32, dev, (n,), "first"),
                                   _dense(last, i32, dev, (n,), "last"), k, ws.data_ptr(), self._stream()), "map_cache_evict")

    def status(self, stream=None) -> int:
        dev = self.device
        if stream is not None or dev.index != _current_device():
            with _on(dev, stream):
                return self.status()
        return lib.map_cache_status(self.desc, _current_stream(dev.index))

    def check(self, stream=None) -> None:
        _check(self.status(stream), "map_cache_status")
