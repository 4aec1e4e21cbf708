"""Thin ctypes binding of libsubgen.so (declared in include/subgen.h).

Argument marshalling only: every step of the path runs in the library's CUDA kernels (the paged functions are called
through the C++ module _calls.so instead of ctypes). torch is used
for device memory and streams. There is no CPU path: loading fails loudly if the shared library is
missing, and every call fails if no CUDA device is usable.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsubgen.so")

DTYPE_FP32, DTYPE_BF16 = 0, 1
ST_CAPACITY, ST_RANGE, ST_TIMEOUT, ST_PAGE, ST_SIZE = 1, 2, 4, 8, 16
STEP_MODES = {"auto": 0, "fused": 1, "split": 2}

EXPORTS = [
    "subgen_workspace_bytes", "subgen_create", "subgen_create_ex", "subgen_destroy", "subgen_prefill",
    "subgen_prefill_varlen", "subgen_step", "subgen_step_host", "subgen_status", "subgen_export_state",
    "subgen_export_rows", "subgen_cache_stats", "subgen_profile_enable", "subgen_profile_read", "subgen_profile_prefill_read",
    "subgen_query", "subgen_launch_count", "subgen_step_kernels", "subgen_last_error", "subgen_checkpoint_bytes", "subgen_checkpoint_save", "subgen_checkpoint_load", "subgen_grow", "subgen_exact_create", "subgen_exact_destroy",
    "subgen_exact_append", "subgen_exact_append_varlen", "subgen_exact_step", "subgen_exact_bytes",
    "subgen_exact_launch_count", "subgen_exact_attention_noalloc",
    "subgen_exact_kcenter_compress", "subgen_exact_kcenter_counters", "subgen_exact_export_tokens",
    "subgen_rope_words", "subgen_qk_norm_rope", "subgen_paged_append", "subgen_paged_workspace_bytes", "subgen_paged_attend",
    "subgen_paged4_append", "subgen_paged4_load", "subgen_paged4_workspace_bytes", "subgen_paged4_attend", "subgen_page_step",
]


class SubgenConfig(C.Structure):
    _fields_ = [("B", C.c_int), ("H", C.c_int), ("Hkv", C.c_int), ("d", C.c_int), ("delta", C.c_float),
                ("t", C.c_int), ("s", C.c_int), ("window", C.c_int), ("seed", C.c_uint64), ("dtype", C.c_int),
                ("m_max", C.c_int), ("splits", C.c_int), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("stream", C.c_void_p), ("nq_max", C.c_int), ("bounded", C.c_int), ("step_mode", C.c_int),
                ("unit_stride", C.c_int), ("unit_offset", C.c_int)]


class StateView(C.Structure):
    _fields_ = [("n", C.c_int), ("inserted", C.c_int), ("m", C.c_int), ("status", C.c_int), ("mu", C.c_uint64),
                ("last_cluster", C.c_int), ("last_opened", C.c_int), ("last_d2", C.c_uint64),
                ("counts", C.c_void_p), ("centre_tok", C.c_void_p), ("slot_tok", C.c_void_p),
                ("m_tok", C.c_void_p), ("m_w", C.c_void_p), ("threshold2", C.c_uint64), ("doublings", C.c_int)]


class Stats(C.Structure):
    _fields_ = [(k, C.c_uint64) for k in ("units", "clusters", "singleton_clusters", "m_filled", "window_rows",
                                           "tokens", "prefill_pairs", "insert_bytes", "query_bytes", "cluster_bytes", "value_bytes",
                                           "distinct_sample_rows")]


class RopeDesc(C.Structure):
    _fields_ = [("words", C.c_void_p), ("rotary_dim", C.c_int), ("interleaved", C.c_int)]


class Heads(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class PagesDesc(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("row_stride", C.c_int64), ("pages", C.c_int), ("page", C.c_int), ("Hkv", C.c_int), ("d", C.c_int),
                ("dtype", C.c_int), ("status", C.c_void_p)]


class Pages4Desc(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("pages", C.c_int), ("page", C.c_int),
                ("Hkv", C.c_int), ("d", C.c_int), ("status", C.c_void_p)]


class BatchDesc(C.Structure):
    _fields_ = [("B", C.c_int), ("cu_q", C.c_void_p), ("lengths", C.c_void_p), ("table", C.c_void_p),
                ("table_stride", C.c_int), ("groups", C.c_int), ("cu_group", C.c_void_p), ("prefix_len", C.c_void_p),
                ("prefix_table", C.c_void_p), ("prefix_stride", C.c_int)]


class QkArgs(C.Structure):
    _fields_ = [(k, Heads) for k in ("q", "k", "v", "q_out", "k_out")] + [
        ("positions", C.c_void_p), ("rope", RopeDesc), ("wq", C.c_void_p), ("wk", C.c_void_p), ("n", C.c_int), ("H", C.c_int),
        ("Hkv", C.c_int), ("d", C.c_int), ("dtype", C.c_int), ("eps", C.c_float), ("fresh", C.c_int)]


class AttendArgs(C.Structure):
    _fields_ = [("q", Heads), ("out", Heads), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("n", C.c_int),
                ("H", C.c_int), ("scale", C.c_float), ("causal", C.c_int), ("fresh", C.c_int)]


class PageStepArgs(C.Structure):
    _fields_ = [("B", C.c_int), ("n", C.c_int), ("pages", C.c_int), ("page", C.c_int), ("table", C.c_void_p), ("table_stride", C.c_int)] + [
        (k, C.c_void_p) for k in ("free_pages", "free_count", "lengths", "added", "ended", "first", "free_count_out", "lengths_out", "cu_q",
                                  "slots", "positions", "status", "sources")]


class SubgenError(RuntimeError):
    pass


_lib = None
_calls = None


def _bind_calls():
    """The calls module (csrc/calls.cpp), which the paged functions go through, over this library. At the first of these calls:
    the rest of the library does without it, whatever torch is installed."""
    global _calls
    L = load()
    from .build import built_for
    advice = "build it with `python paper_2402_06082_b200/build.py`; there is no fallback path"
    try:
        from . import _calls as module
    except ImportError as e:
        raise RuntimeError("_calls.so is missing or was built for another torch: " + advice) from e
    if module.built_for != "built for " + built_for():
        raise RuntimeError("_calls.so was %s, this is %s: %s" % (module.built_for, built_for(), advice))
    at = [C.cast(getattr(L, "subgen_" + f), C.c_void_p).value
          for f in ("qk_norm_rope", "paged_append", "paged_attend", "paged_workspace_bytes", "paged4_append", "paged4_load", "paged4_attend",
                    "paged4_workspace_bytes", "page_step", "last_error")]
    module.bind(SubgenError, *at)
    _calls = module


def load():
    """Load libsubgen.so; raises if it has not been built (python -m paper_2402_06082_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libsubgen.so is missing: build it with `python paper_2402_06082_b200/build.py`; "
                           "there is no fallback path")
    L = C.CDLL(LIB_PATH)
    vp, ip = C.c_void_p, C.POINTER(C.c_int)
    L.subgen_workspace_bytes.restype = C.c_size_t
    L.subgen_workspace_bytes.argtypes = [C.POINTER(SubgenConfig)]
    L.subgen_create.restype = vp
    L.subgen_create.argtypes = [C.c_int, C.c_int, C.c_int, C.c_float, C.c_int, C.c_int, C.c_int, C.c_uint64]
    L.subgen_create_ex.restype = vp
    L.subgen_create_ex.argtypes = [C.POINTER(SubgenConfig)]
    L.subgen_destroy.argtypes = [vp]
    L.subgen_destroy.restype = None
    L.subgen_prefill.argtypes = [vp, vp, vp, C.c_int]
    L.subgen_prefill_varlen.argtypes = [vp, vp, vp, ip]
    L.subgen_step.argtypes = [vp, vp, vp, vp, vp]
    L.subgen_step_host.argtypes = [vp, vp, vp, vp, vp]
    L.subgen_status.argtypes = [vp]
    L.subgen_export_state.argtypes = [vp, C.c_int, C.c_int, C.POINTER(StateView)]
    L.subgen_export_rows.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp, C.c_size_t]
    L.subgen_cache_stats.argtypes = [vp, C.POINTER(Stats)]
    L.subgen_profile_enable.argtypes = [vp, C.c_int]
    L.subgen_profile_read.argtypes = [vp, C.POINTER(C.c_double), ip]
    L.subgen_profile_prefill_read.argtypes = [vp, C.POINTER(C.c_double)]
    L.subgen_launch_count.argtypes = [vp]
    L.subgen_step_kernels.argtypes = [vp]
    L.subgen_query.argtypes = [vp, vp, C.c_int, vp]
    L.subgen_checkpoint_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
    L.subgen_checkpoint_save.argtypes = [vp, vp, C.c_size_t, C.POINTER(C.c_size_t)]
    L.subgen_checkpoint_load.argtypes = [vp, vp, C.c_size_t]
    L.subgen_grow.argtypes = [vp, C.c_int, vp, C.c_size_t]
    L.subgen_launch_count.restype = C.c_uint64
    L.subgen_last_error.restype = C.c_char_p
    L.subgen_exact_create.restype = vp
    L.subgen_exact_create.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, vp]
    L.subgen_exact_destroy.argtypes = [vp]
    L.subgen_exact_destroy.restype = None
    L.subgen_exact_append.argtypes = [vp, vp, vp, C.c_int]
    L.subgen_exact_append_varlen.argtypes = [vp, vp, vp, ip]
    L.subgen_exact_step.argtypes = [vp, vp, vp, vp, vp]
    L.subgen_exact_bytes.argtypes = [vp, C.POINTER(C.c_uint64)]
    L.subgen_exact_launch_count.argtypes = [vp]
    L.subgen_exact_launch_count.restype = C.c_uint64
    L.subgen_exact_kcenter_compress.argtypes = [vp, C.c_int, C.c_int]
    L.subgen_exact_kcenter_counters.argtypes = [vp, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
    L.subgen_exact_export_tokens.argtypes = [vp, C.c_int, C.c_int, ip, ip]
    L.subgen_exact_attention_noalloc.argtypes = [vp, vp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, vp]
    L.subgen_rope_words.argtypes = [C.POINTER(C.c_double), C.c_int, C.POINTER(C.c_uint64)]
    pp, bp = C.POINTER(PagesDesc), C.POINTER(BatchDesc)
    L.subgen_qk_norm_rope.argtypes = [C.POINTER(QkArgs), vp]
    L.subgen_paged_append.argtypes = [pp, bp, C.POINTER(QkArgs), vp]
    L.subgen_paged_workspace_bytes.argtypes = [pp, bp, C.c_int, C.c_int]
    L.subgen_paged_workspace_bytes.restype = C.c_size_t
    L.subgen_paged_attend.argtypes = [pp, bp, C.POINTER(AttendArgs), vp]
    qp = C.POINTER(Pages4Desc)
    L.subgen_paged4_append.argtypes = [qp, bp, C.POINTER(QkArgs), vp]
    L.subgen_paged4_load.argtypes = [qp, vp, C.c_int, C.POINTER(Heads), C.POINTER(Heads), C.c_int, vp]
    L.subgen_paged4_workspace_bytes.argtypes = [qp, bp, C.c_int, C.c_int]
    L.subgen_paged4_workspace_bytes.restype = C.c_size_t
    L.subgen_paged4_attend.argtypes = [qp, bp, C.POINTER(AttendArgs), C.c_int, vp]
    L.subgen_page_step.argtypes = [C.POINTER(PageStepArgs), vp]
    _lib = L
    return L


def _check(rc: int):
    if rc < 0:
        raise SubgenError("subgen error %d: %s" % (rc, load().subgen_last_error().decode()))
    return rc


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return DTYPE_FP32
    if dt == torch.bfloat16:
        return DTYPE_BF16
    raise ValueError("dtype must be torch.float32 or torch.bfloat16")


def _dev(x: torch.Tensor, dt: torch.dtype, shape: Sequence[int], name: str) -> int:
    if not (x.is_cuda and x.is_contiguous() and x.dtype == dt and tuple(x.shape) == tuple(shape)):
        raise ValueError("%s must be a contiguous CUDA %s tensor of shape %s (got %s %s)" %
                         (name, dt, tuple(shape), x.dtype, tuple(x.shape)))
    return x.data_ptr()


class SubGen:
    """One library handle: the SubGen caches of B sequences x Hkv KV heads on the current CUDA device."""

    def __init__(self, B, H, d, delta, t, s, window, seed=0, *, Hkv=None, dtype=torch.bfloat16, m_max=0, splits=0,
                 stream: Optional[torch.cuda.Stream] = None, bounded: bool = False, nq_max: int = 1,
                 step_mode: str = "auto", unit_stride: int = 0, unit_offset: int = 0):
        self._L = load()
        self._h = None
        if not torch.cuda.is_available():
            raise SubgenError("no CUDA device: this library has no CPU path")
        self.bounded = bool(bounded)
        self.B, self.H, self.Hkv, self.d = int(B), int(H), int(Hkv or H), int(d)
        self.t, self.s, self.window, self.dtype = int(t), int(s), int(window), dtype
        self.stream = stream or torch.cuda.current_stream()
        cfg = SubgenConfig(self.B, self.H, self.Hkv, self.d, float(delta), self.t, self.s, self.window, int(seed),
                           _dtype_code(dtype), int(m_max), int(splits), None, 0, self.stream.cuda_stream, int(nq_max), int(bool(bounded)),
                           STEP_MODES[step_mode], int(unit_stride), int(unit_offset))
        nbytes = self._L.subgen_workspace_bytes(C.byref(cfg))
        if nbytes == 0:
            raise SubgenError(self._L.subgen_last_error().decode())
        self._cfg = cfg
        self.m_max = int(m_max) if m_max else 8192
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")   # torch owns the memory
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        cfg.workspace, cfg.workspace_bytes = base, nbytes
        self.workspace_bytes = nbytes
        self._h = self._L.subgen_create_ex(C.byref(cfg))
        if not self._h:
            raise SubgenError(self._L.subgen_last_error().decode())

    def close(self):
        if self._h:
            self._L.subgen_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- stream ---------------------------------------------------------------------------------
    def prefill(self, K: torch.Tensor, V: torch.Tensor):
        n = K.shape[2]
        shp = (self.B, self.Hkv, n, self.d)
        _check(self._L.subgen_prefill(self._h, _dev(K, self.dtype, shp, "K"), _dev(V, self.dtype, shp, "V"), n))

    def prefill_varlen(self, K: torch.Tensor, V: torch.Tensor, cu_seqlens: Sequence[int]):
        cu = (C.c_int * (self.B + 1))(*[int(x) for x in cu_seqlens])
        shp = (self.Hkv, int(cu_seqlens[-1]), self.d)
        _check(self._L.subgen_prefill_varlen(self._h, _dev(K, self.dtype, shp, "K"), _dev(V, self.dtype, shp, "V"), cu))

    def step(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: Optional[torch.Tensor] = None):
        qs, ks = (self.B, self.H, self.d), (self.B, self.Hkv, self.d)
        if out is None:
            out = torch.empty(qs, dtype=self.dtype, device="cuda")
        _check(self._L.subgen_step(self._h, _dev(q, self.dtype, qs, "q"), _dev(k, self.dtype, ks, "k"),
                                   _dev(v, self.dtype, ks, "v"), _dev(out, self.dtype, qs, "out")))
        return out

    def query(self, q: torch.Tensor, out: Optional[torch.Tensor] = None):
        """Read-only QueryStreamAttn for nq queries per head: q [B, H, nq, d] -> out [B, H, nq, d]."""
        nq = int(q.shape[2])
        qs = (self.B, self.H, nq, self.d)
        if out is None:
            out = torch.empty(qs, dtype=self.dtype, device="cuda")
        _check(self._L.subgen_query(self._h, _dev(q, self.dtype, qs, "q"), nq, _dev(out, self.dtype, qs, "out")))
        return out

    def step_host(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor):
        """q, k, v, out are HOST tensors (pinned for asynchronous copies); returns when out is filled."""
        for x in (q, k, v, out):
            if x.is_cuda or not x.is_contiguous() or x.dtype != self.dtype:
                raise ValueError("step_host takes contiguous host tensors of the handle's dtype")
        _check(self._L.subgen_step_host(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr()))
        return out

    def status(self) -> int:
        return _check(self._L.subgen_status(self._h))

    # ---- inspection -----------------------------------------------------------------------------
    def export_state(self, seq: int, kvhead: int) -> dict:
        counts = np.zeros(self.m_max, np.int32)
        ctok = np.zeros(self.m_max, np.int32)
        stok = np.zeros(self.m_max * self.t, np.int32)
        mtok = np.zeros(self.s, np.int32)
        mw = np.zeros(self.s, np.uint64)
        v = StateView()
        v.counts, v.centre_tok, v.slot_tok = counts.ctypes.data, ctok.ctypes.data, stok.ctypes.data
        v.m_tok, v.m_w = mtok.ctypes.data, mw.ctypes.data
        _check(self._L.subgen_export_state(self._h, seq, kvhead, C.byref(v)))
        m = v.m
        return dict(n=v.n, inserted=v.inserted, m=m, status=v.status, mu=int(v.mu), last_cluster=v.last_cluster,
                    last_opened=v.last_opened, last_d2=int(v.last_d2), counts=counts[:m].copy(),
                    centre_tok=ctok[:m].copy(), slot_tok=stok.reshape(self.m_max, self.t)[:m].copy(),
                    m_tok=mtok, m_w=mw, threshold2=int(v.threshold2), doublings=v.doublings)

    def export_rows(self, seq: int, kvhead: int, which: int) -> torch.Tensor:
        rows = {0: self.m_max, 1: self.m_max * self.t, 2: self.s, 3: self.s, 4: self.window, 5: self.window}[which]
        buf = torch.empty((rows, self.d), dtype=self.dtype)
        _check(self._L.subgen_export_rows(self._h, seq, kvhead, which, buf.data_ptr(), buf.numel() * buf.element_size()))
        return buf

    def cache_stats(self) -> dict:
        s = Stats()
        _check(self._L.subgen_cache_stats(self._h, C.byref(s)))
        return {k: int(getattr(s, k)) for k, _ in Stats._fields_}

    def profile_enable(self, on: bool = True):
        _check(self._L.subgen_profile_enable(self._h, int(on)))

    def profile_read(self):
        """(insert_ms, cluster_scan_ms, value_scan_ms, steps) accumulated since the last read."""
        ms, n = (C.c_double * 3)(), C.c_int()
        _check(self._L.subgen_profile_read(self._h, ms, C.byref(n)))
        return ms[0], ms[1], ms[2], n.value

    def profile_prefill_read(self):
        """(value_phase_ms, score_ms, resolve_ms) of the last chunked prefill made with profiling enabled."""
        ms = (C.c_double * 3)()
        _check(self._L.subgen_profile_prefill_read(self._h, ms))
        return ms[0], ms[1], ms[2]

    @property
    def launch_count(self) -> int:
        return int(self._L.subgen_launch_count(self._h))

    @property
    def step_kernels(self) -> int:
        """Kernels one step launches: 1 (fused step), 2 (fp32) or 3."""
        return _check(self._L.subgen_step_kernels(self._h))

    def checkpoint_save(self) -> torch.Tensor:
        """The state between two calls as one pinned uint8 host tensor (see subgen_checkpoint_save)."""
        n = C.c_size_t()
        _check(self._L.subgen_checkpoint_bytes(self._h, C.byref(n)))
        blob = torch.empty(n.value, dtype=torch.uint8, pin_memory=True)
        w = C.c_size_t()
        _check(self._L.subgen_checkpoint_save(self._h, blob.data_ptr(), n.value, C.byref(w)))
        return blob[: w.value]

    def checkpoint_load(self, blob: torch.Tensor):
        """Replace this handle's state by a saved one; the configuration must match, m_max may be larger."""
        if blob.dtype != torch.uint8 or blob.device.type != "cpu" or not blob.is_contiguous():
            raise ValueError("blob must be a contiguous uint8 host tensor")
        _check(self._L.subgen_checkpoint_load(self._h, blob.data_ptr(), blob.numel()))

    def grow(self, m_max: int):
        """Re-lay the state out for a larger cluster capacity per unit (see subgen_grow); the stream continues unchanged."""
        cfg = SubgenConfig.from_buffer_copy(self._cfg)
        cfg.m_max = int(m_max)
        cfg.workspace, cfg.workspace_bytes = None, 0
        nbytes = self._L.subgen_workspace_bytes(C.byref(cfg))
        if nbytes == 0:
            raise SubgenError(self._L.subgen_last_error().decode())
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
        base = (ws.data_ptr() + 255) // 256 * 256
        _check(self._L.subgen_grow(self._h, int(m_max), base, nbytes))
        self.workspace, self.workspace_bytes = ws, nbytes            # the old tensor is released here
        self._cfg.m_max = int(m_max)
        self.m_max = int(m_max)


class ExactAttention:
    """Exact dense decode attention over a full KV cache (Eq. 1), the comparison point."""

    def __init__(self, B, H, d, n_max, *, Hkv=None, dtype=torch.bfloat16, stream: Optional[torch.cuda.Stream] = None):
        self._L = load()
        self._h = None
        if not torch.cuda.is_available():
            raise SubgenError("no CUDA device: this library has no CPU path")
        self.B, self.H, self.Hkv, self.d, self.n_max, self.dtype = int(B), int(H), int(Hkv or H), int(d), int(n_max), dtype
        self.stream = stream or torch.cuda.current_stream()
        self._h = self._L.subgen_exact_create(self.B, self.H, self.Hkv, self.d, self.n_max, _dtype_code(dtype),
                                              self.stream.cuda_stream)
        if not self._h:
            raise SubgenError(self._L.subgen_last_error().decode())

    def close(self):
        if self._h:
            self._L.subgen_exact_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def append(self, K, V):
        n = K.shape[2]
        shp = (self.B, self.Hkv, n, self.d)
        _check(self._L.subgen_exact_append(self._h, _dev(K, self.dtype, shp, "K"), _dev(V, self.dtype, shp, "V"), n))

    def append_varlen(self, K, V, cu_seqlens):
        cu = (C.c_int * (self.B + 1))(*[int(x) for x in cu_seqlens])
        shp = (self.Hkv, int(cu_seqlens[-1]), self.d)
        _check(self._L.subgen_exact_append_varlen(self._h, _dev(K, self.dtype, shp, "K"), _dev(V, self.dtype, shp, "V"), cu))

    def step(self, q, k, v, out=None):
        qs, ks = (self.B, self.H, self.d), (self.B, self.Hkv, self.d)
        if out is None:
            out = torch.empty(qs, dtype=self.dtype, device="cuda")
        _check(self._L.subgen_exact_step(self._h, _dev(q, self.dtype, qs, "q"), _dev(k, self.dtype, ks, "k"),
                                         _dev(v, self.dtype, ks, "v"), _dev(out, self.dtype, qs, "out")))
        return out

    def kcenter_compress(self, k: int, r: int):
        """Keep the r most recent tokens and k greedy k-center centres of the older ones (Section 3.2 variant)."""
        _check(self._L.subgen_exact_kcenter_compress(self._h, int(k), int(r)))

    def kcenter_counters(self):
        """(tokens looked at, full key rows read) of the last compression, summed over units and passes."""
        a, b = C.c_uint64(), C.c_uint64()
        _check(self._L.subgen_exact_kcenter_counters(self._h, C.byref(a), C.byref(b)))
        return int(a.value), int(b.value)

    def export_tokens(self, seq: int, kvhead: int) -> np.ndarray:
        n = C.c_int()
        buf = np.zeros(self.n_max, np.int32)
        _check(self._L.subgen_exact_export_tokens(self._h, seq, kvhead, C.byref(n), buf.ctypes.data_as(C.POINTER(C.c_int))))
        return buf[: n.value].copy()

    def bytes_per_step(self) -> int:
        b = C.c_uint64()
        _check(self._L.subgen_exact_bytes(self._h, C.byref(b)))
        return int(b.value)

    @property
    def launch_count(self) -> int:
        return int(self._L.subgen_exact_launch_count(self._h))


NOALLOC_SCRATCH_BYTES = 4 << 20


def exact_attention_noalloc(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, out: torch.Tensor,
                            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out = softmax(K q)^T V per head without any device allocation by the library.

    For callers that may not call cudaMalloc (a plugin inside a process whose allocator owns all device
    memory, or request-path code that cannot take an allocation's synchronisation): the split partials
    live in a fixed array inside the library image (NOALLOC_SCRATCH_BYTES per GPU, shared by all calls,
    so calls that can overlap on the GPU must be ordered). q, out: CUDA [B, H, d]; K, V: CUDA [B, Hkv, n, d].
    The caller supplies `out`; this wrapper creates no tensor.
    """
    B, H, d = q.shape
    Hkv, n = K.shape[1], K.shape[2]
    dt = q.dtype
    st = stream or torch.cuda.current_stream()
    _check(load().subgen_exact_attention_noalloc(
        _dev(q, dt, (B, H, d), "q"), _dev(K, dt, (B, Hkv, n, d), "K"), _dev(V, dt, (B, Hkv, n, d), "V"),
        _dev(out, dt, (B, H, d), "out"), B, H, Hkv, d, n, _dtype_code(dt), st.cuda_stream))
    return out


# ---- norms, rotation and the paged exact cache --------------------------------------------------
#
# These calls run on the current stream of their tensors' device and keep nothing between calls: outputs and scratch
# come from torch's allocator, call by call, so captured graphs and calls on several streams do not share any. They go
# through the calls module: a step of a small model makes several of them a layer, and ctypes would cost more on the
# host than their kernels take.

def _whole(x: torch.Tensor, name: str, device: int, shape) -> int:
    if x.dtype is not torch.int32 or x.get_device() != device or x.shape != shape or not x.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s on cuda:%d (got %s %s on %s)" %
                         (name, tuple(shape), device, x.dtype, tuple(x.shape), x.device))
    return x.data_ptr()


def _cuda(x: torch.Tensor, name: str) -> int:
    i = x.get_device()
    if i < 0:
        raise ValueError("%s must be a CUDA tensor: this library has no CPU path" % name)
    return i


class Rope:
    """Position rotation of the first `rotary_dim` of d coordinates: pairs (i, i + r/2), or (2i, 2i + 1) if interleaved.

    Pair i turns by base^(-2i/r) radians per position, or by inv_freq[i] where r/2 values are given (scaled variants).
    """

    def __init__(self, d: int, base: float = 10000.0, rotary_dim: Optional[int] = None, interleaved: bool = False,
                 inv_freq: Optional[Sequence[float]] = None, device="cuda"):
        r = int(d if rotary_dim is None else rotary_dim)
        if r <= 0 or r > d or r % 16:
            raise ValueError("rotary_dim must be a multiple of 16 and at most d")
        f = [float(base) ** (-2.0 * i / r) for i in range(r // 2)] if inv_freq is None else [float(x) for x in inv_freq]
        if len(f) != r // 2:
            raise ValueError("inv_freq must hold rotary_dim / 2 values")
        words = np.zeros(r // 2, np.uint64)
        _check(load().subgen_rope_words((C.c_double * (r // 2))(*f), r // 2, words.ctypes.data_as(C.POINTER(C.c_uint64))))
        self.d, self.rotary_dim, self.interleaved = int(d), r, bool(interleaved)
        self.words = torch.from_numpy(words.view(np.int64)).to(device)
        self._desc = (self.words.data_ptr(), r, int(self.interleaved), self.d, self.words.get_device())


def qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                 rope: Optional[Rope] = None, *, wq: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """RMS norm of every head (where a weight is given), then the rotation by `positions` (int32 [n]); see subgen_qk_norm_rope.

    q [n, H, d], k [n, Hkv, d]: views with unit stride along d (slices of a fused projection). Returns (q_out, k_out), None for
    what was not given; an output may be its input.
    """
    if _calls is None:
        _bind_calls()
    return _calls.qk_norm_rope(q, k, positions, None if rope is None else rope._desc, wq, wk, eps, q_out, k_out)


class PagedBatch:
    """The sequences of a call on a PagedCache (see subgen_batch): int32 CUDA tensors, kept and read by every call.

    cu_q [B + 1]: rows cu_q[b] .. cu_q[b + 1] of q, k, v are the new tokens of sequence b, the last of its lengths[b] own
    tokens; table [B, m]: the pages of each. cu_group [g + 1], prefix_len [g], prefix_table [g, m']: sequences cu_group[i] ..
    cu_group[i + 1] share the prefix_len[i] tokens in prefix_table[i]. Contents may change between calls (and replays).
    """

    def __init__(self, cu_q: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, cu_group: Optional[torch.Tensor] = None,
                 prefix_len: Optional[torch.Tensor] = None, prefix_table: Optional[torch.Tensor] = None):
        dev = self.device = _cuda(lengths, "lengths")
        B = self.B = int(lengths.shape[0])
        given = [x is not None for x in (cu_group, prefix_len, prefix_table)]
        if any(given) != all(given):
            raise ValueError("cu_group, prefix_len and prefix_table come together")
        g = int(prefix_len.shape[0]) if all(given) else 0
        if table.dim() != 2 or (g and prefix_table.dim() != 2):
            raise ValueError("page tables are two-dimensional")
        self.tensors = (cu_q, lengths, table, cu_group, prefix_len, prefix_table)
        self._desc = BatchDesc(B, _whole(cu_q, "cu_q", dev, (B + 1,)), _whole(lengths, "lengths", dev, (B,)),
                               _whole(table, "table", dev, (B, table.shape[1])), table.shape[1], g)
        if g:
            self._desc.cu_group = _whole(cu_group, "cu_group", dev, (g + 1,))
            self._desc.prefix_len = _whole(prefix_len, "prefix_len", dev, (g,))
            self._desc.prefix_table = _whole(prefix_table, "prefix_table", dev, (g, prefix_table.shape[1]))
            self._desc.prefix_stride = prefix_table.shape[1]
        self._at = C.addressof(self._desc)


class PagedCache:
    """An exact cache in pages: K, V [pages, Hkv, page, d], owned by the caller (any strides with unit stride along d, the
    same for both, so that [pages, page, Hkv, d] pools and halves of one tensor serve as well). See subgen_pages."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor):
        dev = self.device = _cuda(K, "K")
        if K.dim() != 4 or K.stride(3) != 1 or V.shape != K.shape or V.stride() != K.stride() or V.dtype is not K.dtype or V.get_device() != dev:
            raise ValueError("K and V must be [pages, Hkv, page, d] tensors of one type, device and layout, unit stride along d")
        if _calls is None:
            _bind_calls()
        self.K, self.V, self.dtype = K, V, K.dtype
        self.pages, self.Hkv, self.page, self.d = K.shape
        self._status = torch.zeros(1, dtype=torch.int32, device=K.device)
        if not torch.cuda.is_current_stream_capturing():   # 0 before a call on any stream may set a bit (made once a pool)
            torch.cuda.current_stream(dev).synchronize()
        self._desc = PagesDesc(K.data_ptr(), V.data_ptr(), K.stride(0), K.stride(1), K.stride(2), self.pages, self.page, self.Hkv,
                               self.d, _dtype_code(K.dtype), self._status.data_ptr())
        self._at = C.addressof(self._desc)

    def _batch(self, batch: PagedBatch) -> int:
        if batch.device != self.device:
            raise ValueError("the batch is on device %d, the cache on %d" % (batch.device, self.device))
        return batch._at

    def append(self, batch: PagedBatch, k: torch.Tensor, v: torch.Tensor, *, rope: Optional[Rope] = None,
               positions: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None, eps: float = 1e-6,
               q: Optional[torch.Tensor] = None, wq: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
        """Write the new tokens k, v [n, Hkv, d] into their pages, k normed (if wk) and rotated (if rope) on the way; q [n, H, d]
        goes the same way into q_out, which is returned (None without q). A token that broken offsets or groups leave out (status())
        keeps its row of a q_out that was given, and is NaN in a new one. One kernel; see subgen_paged_append."""
        return _calls.append(self._at, self.device, self._batch(batch), k, v, positions, None if rope is None else rope._desc, wk, eps,
                             q, wq, q_out)

    def attend(self, batch: PagedBatch, q: torch.Tensor, scale: float = 1.0, causal: bool = True, out: Optional[torch.Tensor] = None):
        """softmax(scale q [Kprefix; Kown]^T) [Vprefix; Vown] for q [n, H, d], whose keys are in the cache already; a prefix is
        read for the rows of its group's sequences together. Rows of `out` behind the last sequence are not written (of a new
        one: undefined). Broken offsets and batches that are too long leave an `out` that was given as it is and make NaN of a
        new one; status() tells. See subgen_paged_attend."""
        return _calls.attend(self._at, self.device, self._batch(batch), q, scale, causal, out)

    def status(self) -> int:
        """Waits for the device's work, returns the status bits that calls on this cache have set (0: none)."""
        torch.cuda.synchronize(self.device)
        return int(self._status.item())


class PagedCache4:
    """A cache in pages that holds keys and values in 4 bits, 4.5 with their scales (see subgen_pages4): pool [pages, Hkv, bytes] uint8
    with bytes(page, d) on end for each head, owned by the caller (any strides of pages and heads, multiples of 16). Takes fp32 and bf16
    queries, keys and values, call by call. (Made while a stream captures, every replay begins with a status of 0.)"""

    def __init__(self, pool: torch.Tensor, page: int, d: int):
        dev = self.device = _cuda(pool, "pool")
        if pool.dtype is not torch.uint8 or pool.dim() != 3 or pool.stride(2) != 1 or pool.shape[2] != self.bytes(page, d):
            raise ValueError("pool must be a uint8 tensor [pages, Hkv, %d] with unit stride along the last axis (got %s %s)" %
                             (self.bytes(page, d), pool.dtype, tuple(pool.shape)))
        if _calls is None:
            _bind_calls()
        self.pool, self.page, self.d = pool, int(page), int(d)
        self.pages, self.Hkv = pool.shape[:2]
        self._status = torch.zeros(1, dtype=torch.int32, device=pool.device)
        if not torch.cuda.is_current_stream_capturing():   # 0 before a call on any stream may set a bit (made once a pool)
            torch.cuda.current_stream(dev).synchronize()
        self._desc = Pages4Desc(pool.data_ptr(), pool.stride(0), pool.stride(1), self.pages, self.page, self.Hkv, self.d, self._status.data_ptr())
        self._at = C.addressof(self._desc)

    @staticmethod
    def bytes(page: int, d: int) -> int:
        """What a page takes in one head: codes and scales of its keys and values."""
        return int(page) * 2 * (int(d) // 2 + int(d) // 16)

    def _batch(self, batch: PagedBatch) -> int:
        if batch.device != self.device:
            raise ValueError("the batch is on device %d, the cache on %d" % (batch.device, self.device))
        return batch._at

    def append(self, batch: PagedBatch, k: torch.Tensor, v: torch.Tensor, *, rope: Optional[Rope] = None,
               positions: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None, eps: float = 1e-6,
               q: Optional[torch.Tensor] = None, wq: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
        """PagedCache.append with keys and values rounded to 4 bits on the way. One kernel; see subgen_paged4_append."""
        return _calls.append4(self._at, self.device, self._batch(batch), k, v, positions, None if rope is None else rope._desc, wk, eps,
                              q, wq, q_out)

    def attend(self, batch: PagedBatch, q: torch.Tensor, scale: float = 1.0, causal: bool = True, out: Optional[torch.Tensor] = None):
        """PagedCache.attend over the values that the cells stand for. See subgen_paged4_attend."""
        return _calls.attend4(self._at, self.device, self._batch(batch), q, scale, causal, out)

    def load(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None):
        """Keys and values [n, Hkv, d] of the tokens in `slots` (int64, page * tokens per page + row; below 0: zeros), exact: what a
        SubGen.prefill or an exact cache takes. K, V: outputs, views with unit stride along d. See subgen_paged4_load."""
        return _calls.load4(self._at, self.device, slots, _dtype_code(dtype), K, V)

    def status(self) -> int:
        """Waits for the device's work, returns the status bits that calls on this cache have set (0: none)."""
        torch.cuda.synchronize(self.device)
        return int(self._status.item())


class PageStep(NamedTuple):
    """What page_step gives: cu_q [B + 1], lengths [B], free_count [1], slots [n] (int64; -1 behind the last token), positions [n]."""
    cu_q: torch.Tensor
    lengths: torch.Tensor
    free_count: torch.Tensor
    slots: torch.Tensor
    positions: torch.Tensor


def page_step(lengths: torch.Tensor, table: torch.Tensor, free: torch.Tensor, free_count: torch.Tensor, added: torch.Tensor, page: int, n: int,
              *, ended: Optional[torch.Tensor] = None, first: Optional[torch.Tensor] = None, in_place: bool = True, cu_q: Optional[torch.Tensor] = None,
              slots: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
              sources: Optional[torch.Tensor] = None) -> PageStep:
    """The tables of a step, on the device (see subgen_page_step): rows that ended give their pages back, rows with new tokens get pages.

    lengths, added, ended, first [B], table [B, m], free [pages], free_count, status [1]: int32. The table and the stack of free pages change
    in place; lengths and free_count too, or (in_place=False) into new tensors. n: rows of the step's tensors, which slots and positions are
    made for. added may ask for more than there is: rows that are not served get no new tokens, and those of the rows behind them move up. sources
    (int32 [n], an output) then tells which of the tokens that were asked for each one is: inputs that lie by `added` are taken by it.
    """
    if _calls is None:
        _bind_calls()
    return PageStep(*_calls.page_step(lengths, table, free, free_count, added, page, n, ended, first, lengths if in_place else None,
                                      free_count if in_place else None, cu_q, slots, positions, status, sources))


class PageTables:
    """Lengths, page tables and free pages of B requests over a pool, kept on the device, and the batch that a paged cache's calls take.

    step() serves a step's new tokens and moves on; a captured graph may hold it and the calls behind it, since batch, slots, positions and
    sources stay where they are. A row that is not served (status()) gets nothing, and what is behind it moves up: q[tables.sources] are the
    rows of a q that holds all tokens that were asked for, [n, ...] (its row 0 behind the last).
    A row's request is over when `ended` says so, and the row is free for the next one, in the same step if it has to be.
    Make it before a capture. Made while a stream captures, its empty tables are a part of the graph: it holds nothing before the first replay, and
    every replay begins with no tokens and all pages free.
    """

    def __init__(self, B: int, pages_per_row: int, pages: int, page: int, n: int, device="cuda"):
        ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=device)  # noqa: E731
        self.page, self.n = int(page), int(n)
        self.lengths, self.table, self.cu_q, self._status = ints(B), ints(B, pages_per_row), ints(B + 1), ints(1)
        self.free = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device)      # page 0 is on top
        self.free_count = torch.full((1,), pages, dtype=torch.int32, device=device)
        self.slots, self.positions, self.sources = torch.full((self.n,), -1, dtype=torch.int64, device=device), ints(self.n), ints(self.n)
        self.batch = PagedBatch(self.cu_q, self.lengths, self.table)
        if not torch.cuda.is_current_stream_capturing():   # as they are before a call on any stream reads them
            torch.cuda.current_stream(self.lengths.device).synchronize()

    def step(self, added: torch.Tensor, ended: Optional[torch.Tensor] = None) -> PageStep:
        """added [B]: the tokens that each request gets now; ended [B]: nonzero where a request is over (both int32). What is given back is
        what the object holds: the next step changes it."""
        return page_step(self.lengths, self.table, self.free, self.free_count, added, self.page, self.n, ended=ended, cu_q=self.cu_q,
                         slots=self.slots, positions=self.positions, status=self._status, sources=self.sources)

    def status(self) -> int:
        """Waits for the device's work, returns the status bits that steps have set: ST_CAPACITY where a row was not served (0: none)."""
        torch.cuda.synchronize(self.lengths.device)
        return int(self._status.item())
