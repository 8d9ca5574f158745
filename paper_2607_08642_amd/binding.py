"""Thin Python binding of libdominotree (include/dominotree.h).

Argument marshalling only: every step of the tree build runs in the HIP
kernels behind the C ABI.  torch is used for device memory and streams.  The
library is loaded from this package directory; if it is missing, every call
raises (there is no fallback).
"""
from __future__ import annotations

import ctypes
import dataclasses
import operator
import os
import threading
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libdominotree.so")

DT_F32 = 0
DT_BF16 = 1
DT_F8 = 2
DT_NORM_TAIL = 0
DT_NORM_SLICE = 1
DT_SCORER_COND = 0
DT_SCORER_MARG = 1
DT_SCORER_STATIC = 2
DT_TREE_NONFINITE = 0x1
DT_TREE_TRUNCATED = 0x2
DT_TREE_TIMEOUT = 0x4
ABI_VERSION = 3

STATUS = {0: "DT_OK", -1: "DT_ERR_NULL", -2: "DT_ERR_SHAPE", -3: "DT_ERR_DTYPE",
          -4: "DT_ERR_UNSUPPORTED", -5: "DT_ERR_WORKSPACE", -6: "DT_ERR_ALIGN", -7: "DT_ERR_HIP"}

# every symbol include/dominotree.h declares
EXPORTS = ("dt_abi_version", "dt_status_string", "dt_last_error", "dt_plan_create",
           "dt_workspace_size", "dt_build_tree", "dt_plan_destroy", "dt_plan_set_profiling",
           "dt_plan_stage_ms", "dt_scan_workspace_size", "dt_scan_topm", "dt_head_workspace_size",
           "dt_build_tree_head", "dt_build_tree_noalloc",
           "dt_plan_expand_stats", "dt_plan_set_adaptive_budget", "dt_model_create",
           "dt_model_destroy", "dt_plan_create_from_model", "dt_once_workspace_size",
           "dt_build_tree_once", "dt_cache_size", "dt_cache_append", "dt_cache_read",
           "dt_attend_workspace_size", "dt_cache_attend", "dt_tree_accept", "dt_cache_commit",
           "dt_rotate", "dt_cache_append_rotated", "dt_sample_workspace_size", "dt_sample",
           "dt_pages_workspace_size", "dt_pages_fit", "dt_pages_fork", "dt_pages_compact", "dt_cache_copy_pages")
STAGES = ("scan", "expand")


class DTError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class dt_gru(ctypes.Structure):
    _fields_ = [("w_ih", ctypes.c_void_p), ("w_hh", ctypes.c_void_p), ("b_ih", ctypes.c_void_p),
                ("b_hh", ctypes.c_void_p), ("d_in", ctypes.c_int), ("d_h", ctypes.c_int)]


class dt_head(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("b", ctypes.c_void_p)]


class dt_domino_head(ctypes.Structure):
    _fields_ = [("w1", ctypes.c_void_p), ("w2", ctypes.c_void_p), ("d_H", ctypes.c_int),
                ("rank", ctypes.c_int)]


class dt_options(ctypes.Structure):
    _fields_ = [("max_children", ctypes.c_int), ("norm_mode", ctypes.c_int),
                ("pos_offset", ctypes.c_int), ("scorer", ctypes.c_int),
                ("frontier_width", ctypes.c_int), ("debug_spin_limit", ctypes.c_int)]


class dt_tree(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("parents", ctypes.c_void_p),
                ("depth", ctypes.c_void_p), ("position_ids", ctypes.c_void_p),
                ("mask", ctypes.c_void_p), ("scores", ctypes.c_void_p),
                ("n_nodes", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class dt_cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("layers", ctypes.c_int), ("pages", ctypes.c_int),
                ("page_size", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("dtype", ctypes.c_int)]


class dt_chunk(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("rows", ctypes.c_int), ("max_chunk", ctypes.c_int),
                ("max_len", ctypes.c_int), ("table_width", ctypes.c_int), ("starts", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("table", ctypes.c_void_p)]


class dt_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class dt_attend_options(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("window", ctypes.c_int), ("sinks", ctypes.c_int),
                ("tree_nodes", ctypes.c_int), ("mask", ctypes.c_void_p), ("depth", ctypes.c_void_p)]


class dt_rotary(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p), ("pairs", ctypes.c_int),
                ("interleaved", ctypes.c_int), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float)]


class dt_sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("top_k", ctypes.c_int), ("temperatures", ctypes.c_void_p), ("top_ps", ctypes.c_void_p),
                ("min_ps", ctypes.c_void_p), ("top_ks", ctypes.c_void_p)]


class dt_pages(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int), ("page_size", ctypes.c_int), ("batch", ctypes.c_int),
                ("table_width", ctypes.c_int), ("uses", ctypes.c_void_p), ("held", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("table", ctypes.c_void_p), ("missing", ctypes.c_void_p)]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the shared library (raises if it is missing or its ABI differs)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2607_08642_amd.build.build()")
    lib = ctypes.CDLL(path)
    vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.dt_abi_version.restype = ci
    lib.dt_status_string.restype = ctypes.c_char_p
    lib.dt_status_string.argtypes = [ci]
    lib.dt_last_error.restype = ctypes.c_char_p
    lib.dt_plan_create.restype = ci
    lib.dt_plan_create.argtypes = [ctypes.POINTER(vp), vp, ci, ci, ctypes.POINTER(dt_gru),
                                   ctypes.POINTER(dt_head), ci, ci, ci, ci, ci, ci,
                                   ctypes.POINTER(dt_options)]
    lib.dt_model_create.restype = ci
    lib.dt_model_create.argtypes = [ctypes.POINTER(vp), vp, ci, ci, ctypes.POINTER(dt_gru),
                                    ctypes.POINTER(dt_head), ci]
    lib.dt_model_destroy.restype = None
    lib.dt_model_destroy.argtypes = [vp]
    lib.dt_plan_create_from_model.restype = ci
    lib.dt_plan_create_from_model.argtypes = [ctypes.POINTER(vp), vp, ci, ci, ci, ci, ci,
                                              ctypes.POINTER(dt_options)]
    lib.dt_workspace_size.restype = ci
    lib.dt_workspace_size.argtypes = [vp, ci, ctypes.POINTER(sz)]
    lib.dt_build_tree.restype = ci
    lib.dt_build_tree.argtypes = [vp, vp, ci, vp, cf, vp, sz, ctypes.POINTER(dt_tree), vp]
    lib.dt_plan_destroy.restype = None
    lib.dt_plan_destroy.argtypes = [vp]
    lib.dt_plan_set_profiling.restype = ci
    lib.dt_plan_set_profiling.argtypes = [vp, ci]
    lib.dt_plan_stage_ms.restype = ci
    lib.dt_plan_stage_ms.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
    lib.dt_scan_workspace_size.restype = ci
    lib.dt_scan_workspace_size.argtypes = [ci, ci, ci, ctypes.POINTER(sz)]
    lib.dt_scan_topm.restype = ci
    lib.dt_head_workspace_size.restype = ci
    lib.dt_head_workspace_size.argtypes = [vp, ci, ctypes.POINTER(dt_domino_head), ctypes.POINTER(sz)]
    lib.dt_build_tree_head.restype = ci
    lib.dt_build_tree_head.argtypes = [vp, vp, ci, vp, ctypes.POINTER(dt_domino_head), vp, cf, vp,
                                       sz, ctypes.POINTER(dt_tree), vp]
    lib.dt_scan_topm.argtypes = [vp, ci, ci, ci, ci, cf, vp, vp, vp, vp, vp, sz, vp]
    lib.dt_plan_set_adaptive_budget.restype = ci
    lib.dt_plan_set_adaptive_budget.argtypes = [vp, cf, ctypes.POINTER(cf), ci]
    lib.dt_plan_expand_stats.restype = ci
    lib.dt_plan_expand_stats.argtypes = [vp, vp, vp, ci]
    lib.dt_build_tree_noalloc.restype = ci
    lib.dt_build_tree_noalloc.argtypes = [vp, vp, ci, vp, cf, ctypes.POINTER(dt_tree), vp]
    lib.dt_once_workspace_size.restype = ci
    lib.dt_once_workspace_size.argtypes = [ci] * 9 + [ctypes.POINTER(dt_options), ctypes.POINTER(sz)]
    lib.dt_build_tree_once.restype = ci
    lib.dt_build_tree_once.argtypes = [vp, ci, ci, ctypes.POINTER(dt_gru), ctypes.POINTER(dt_head)] + [ci] * 5 + \
        [vp, ci, vp, cf, ctypes.POINTER(dt_options), vp, sz, ctypes.POINTER(dt_tree), vp]
    pc, pk, pr, po = (ctypes.POINTER(t) for t in (dt_cache, dt_chunk, dt_rows, dt_attend_options))
    lib.dt_cache_size.restype = ci
    lib.dt_cache_size.argtypes = [pc, ctypes.POINTER(sz)]
    for f in (lib.dt_cache_append, lib.dt_cache_read):
        f.restype = ci
        f.argtypes = [pc, ci, pk, pr, pr, vp]
    lib.dt_attend_workspace_size.restype = ci
    lib.dt_attend_workspace_size.argtypes = [pc, pk, ci, po, ctypes.POINTER(sz)]
    lib.dt_cache_attend.restype = ci
    lib.dt_cache_attend.argtypes = [pc, ci, pk, ci, pr, pr, po, vp, sz, vp]
    lib.dt_tree_accept.restype = ci
    lib.dt_tree_accept.argtypes = [ctypes.POINTER(dt_tree), ci, ci, vp, vp, vp, vp, vp]
    lib.dt_cache_commit.restype = ci
    lib.dt_cache_commit.argtypes = [pc, pk, ci, vp, vp, vp]
    pt = ctypes.POINTER(dt_rotary)
    lib.dt_rotate.restype = ci
    lib.dt_rotate.argtypes = [pr, ci, pr, ci, ci, ci, ci, pt, pr, pr, vp]
    lib.dt_cache_append_rotated.restype = ci
    lib.dt_cache_append_rotated.argtypes = [pc, ci, pk, ci, pr, pr, pr, pt, pr, vp]
    lib.dt_sample_workspace_size.restype = ci
    lib.dt_sample_workspace_size.argtypes = [ci, ci, ctypes.POINTER(sz)]
    lib.dt_sample.restype = ci
    lib.dt_sample.argtypes = [vp, ctypes.c_int64, ci, ci, ci, vp, ctypes.POINTER(dt_sampling), vp, vp, vp, sz, vp]
    pg = ctypes.POINTER(dt_pages)
    lib.dt_pages_workspace_size.restype = ci
    lib.dt_pages_workspace_size.argtypes = [pg, ctypes.POINTER(sz)]
    lib.dt_pages_fit.restype = ci
    lib.dt_pages_fit.argtypes = [pg, vp, sz, vp]
    lib.dt_pages_fork.restype = ci
    lib.dt_pages_fork.argtypes = [pg, pc, vp, vp, sz, vp]
    lib.dt_pages_compact.restype = ci
    lib.dt_pages_compact.argtypes = [pg, pc, vp, sz, vp]
    lib.dt_cache_copy_pages.restype = ci
    lib.dt_cache_copy_pages.argtypes = [pc, vp, vp, ci, vp]
    if lib.dt_abi_version() != ABI_VERSION:
        raise RuntimeError(f"ABI mismatch: library {lib.dt_abi_version()} vs binding {ABI_VERSION}")
    _lib = lib
    return lib


def _check(st: int) -> None:
    if st != 0:
        raise DTError(st, load().dt_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return DT_BF16
    if t.dtype == torch.float32:
        return DT_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream) -> Optional[int]:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


@dataclasses.dataclass
class Tree:
    """Emitted trees (device tensors), nodes in pop order."""
    tokens: "torch.Tensor"        # [b, B] int32
    parents: "torch.Tensor"       # [b, B] int32, -1 = child of the root
    depth: "torch.Tensor"         # [b, B] int32
    position_ids: "torch.Tensor"  # [b, B] int32
    mask: "torch.Tensor"          # [b, B, B] uint8 ancestor-or-self
    scores: "torch.Tensor"        # [b, B] float32
    n_nodes: "torch.Tensor"       # [b] int32
    status: "torch.Tensor"        # [b] int32

    @staticmethod
    def empty(batch: int, B: int, device) -> "Tree":
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        return Tree(torch.empty(batch, B, **i32), torch.empty(batch, B, **i32),
                    torch.empty(batch, B, **i32), torch.empty(batch, B, **i32),
                    torch.empty(batch, B, B, dtype=torch.uint8, device=device),
                    torch.empty(batch, B, dtype=torch.float32, device=device),
                    torch.empty(batch, **i32), torch.empty(batch, **i32))

    def as_c(self) -> dt_tree:
        """The dt_tree view of these tensors (built once; the tensors never move)."""
        c = self.__dict__.get("_c")
        if c is None:
            c = dt_tree(*(x.data_ptr() for x in (self.tokens, self.parents, self.depth,
                                                    self.position_ids, self.mask, self.scores,
                                                    self.n_nodes, self.status)))
            self.__dict__["_c"] = c
        return c


class Model:
    """dt_model: a drafter's vocabulary tables (embedding table folded through
    the GRU input projection and the correction head) and repacked GRU, shared
    by every Plan made from it.  The weight tensors may be freed once it exists.
    """

    def __init__(self, emb, w_ih, w_hh, b_ih, b_hh, w_c, b_c):
        lib = load()
        self._lib = lib
        self.V, self.d_e = emb.shape
        self.d_h = w_hh.shape[1]
        self.device = emb.device
        gru = dt_gru(_ptr(w_ih), _ptr(w_hh), _ptr(b_ih), _ptr(b_hh), self.d_e, self.d_h)
        head = dt_head(_ptr(w_c), _ptr(b_c))
        h = ctypes.c_void_p()
        _check(lib.dt_model_create(ctypes.byref(h), _ptr(emb), self.V, self.d_e, ctypes.byref(gru),
                                   ctypes.byref(head), _dtype_code(emb)))
        self.handle = h

    def close(self) -> None:
        """Drop this reference (the tables live on while a plan uses them)."""
        if getattr(self, "handle", None):
            self._lib.dt_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Plan:
    """dt_plan: one model (embedding table, GRU, head) and one (L, M, B) shape.

    Plan(emb, w_ih, ...) builds a model of its own (dt_plan_create);
    Plan.from_model(model, ...) shares an existing Model's tables.
    """

    def __init__(self, emb, w_ih, w_hh, b_ih, b_hh, w_c, b_c, *, L: int, M: int, B: int,
                 logits_dtype: int, max_batch: int = 1, max_children: int = 0,
                 norm_mode: int = DT_NORM_TAIL, pos_offset: int = 0,
                 scorer: int = DT_SCORER_COND, frontier_width: int = 0,
                 debug_spin_limit: int = 0):
        lib = load()
        self._lib = lib
        self.V, self.d_e = emb.shape
        self.d_h = w_hh.shape[1]
        self.device = emb.device
        self.L, self.M, self.B, self.max_batch = L, M, B, max_batch
        self.logits_dtype = logits_dtype
        wdt = _dtype_code(emb)
        gru = dt_gru(_ptr(w_ih), _ptr(w_hh), _ptr(b_ih), _ptr(b_hh), self.d_e, self.d_h)
        head = dt_head(_ptr(w_c), _ptr(b_c))
        opts = dt_options(max_children, norm_mode, pos_offset, scorer, frontier_width,
                          debug_spin_limit)
        h = ctypes.c_void_p()
        _check(lib.dt_plan_create(ctypes.byref(h), _ptr(emb), self.V, self.d_e, ctypes.byref(gru),
                                  ctypes.byref(head), wdt, L, M, B, logits_dtype, max_batch,
                                  ctypes.byref(opts)))
        self.handle = h
        self._ws = {}

    @classmethod
    def from_model(cls, model: Model, *, L: int, M: int, B: int, logits_dtype: int,
                   max_batch: int = 1, max_children: int = 0, norm_mode: int = DT_NORM_TAIL,
                   pos_offset: int = 0, scorer: int = DT_SCORER_COND, frontier_width: int = 0,
                   debug_spin_limit: int = 0) -> "Plan":
        """dt_plan_create_from_model: a plan over `model`'s tables."""
        self = cls.__new__(cls)
        self._lib = model._lib
        self.V, self.d_e, self.d_h, self.device = model.V, model.d_e, model.d_h, model.device
        self.L, self.M, self.B, self.max_batch = L, M, B, max_batch
        self.logits_dtype = logits_dtype
        opts = dt_options(max_children, norm_mode, pos_offset, scorer, frontier_width,
                          debug_spin_limit)
        h = ctypes.c_void_p()
        _check(self._lib.dt_plan_create_from_model(ctypes.byref(h), model.handle, L, M, B,
                                                   logits_dtype, max_batch, ctypes.byref(opts)))
        self.handle = h
        self._ws = {}
        return self

    def workspace_size(self, batch: int) -> int:
        n = ctypes.c_size_t()
        _check(self._lib.dt_workspace_size(self.handle, batch, ctypes.byref(n)))
        return n.value

    def workspace(self, batch: int):
        import torch
        if batch not in self._ws:
            self._ws[batch] = torch.empty(self.workspace_size(batch), dtype=torch.uint8,
                                          device=self.device)
        return self._ws[batch]

    def build_tree(self, logits, T: float, h0=None, out: Optional[Tree] = None,
                   workspace=None, stream=None) -> Tree:
        """dt_build_tree on torch's current stream (asynchronous)."""
        batch = logits.shape[0]
        if out is None:
            out = Tree.empty(batch, self.B, logits.device)
        ws = self.workspace(batch) if workspace is None else workspace
        st = self._lib.dt_build_tree(self.handle, logits.data_ptr(), batch,
                                     None if h0 is None else h0.data_ptr(), T, ws.data_ptr(),
                                     ws.numel(), ctypes.byref(out.as_c()), _stream(stream))
        if st != 0:
            _check(st)
        return out

    def build_tree_noalloc(self, logits, T: float, h0=None, out: Optional[Tree] = None,
                           stream=None) -> Tree:
        """dt_build_tree_noalloc: no workspace argument (the library's per-device
        scratch array); `out` must be given by callers that cannot allocate."""
        batch = logits.shape[0]
        if out is None:
            out = Tree.empty(batch, self.B, logits.device)
        st = self._lib.dt_build_tree_noalloc(self.handle, logits.data_ptr(), batch,
                                             None if h0 is None else h0.data_ptr(), T,
                                             ctypes.byref(out.as_c()), _stream(stream))
        if st != 0:
            _check(st)
        return out

    def _head(self, w1, w2) -> dt_domino_head:
        rank, width = w1.shape
        return dt_domino_head(_ptr(w1), _ptr(w2), width - self.d_h, rank)

    def head_workspace_size(self, batch: int, w1, w2) -> int:
        n = ctypes.c_size_t()
        hd = self._head(w1, w2)
        _check(self._lib.dt_head_workspace_size(self.handle, batch, ctypes.byref(hd), ctypes.byref(n)))
        return n.value

    def build_tree_head(self, logits, H, w1, w2, T: float, h0=None, out: Optional[Tree] = None,
                        workspace=None, stream=None) -> Tree:
        """dt_build_tree_head (Domino's own head: w1 [rank, d_H + d_h], w2 [V, rank],
        H [b, L, d_H], all in the weights dtype) on torch's current stream."""
        import torch
        batch = logits.shape[0]
        if out is None:
            out = Tree.empty(batch, self.B, logits.device)
        hd = self._head(w1, w2)
        if workspace is None:
            key = ("head", batch, hd.rank)
            if key not in self._ws:
                self._ws[key] = torch.empty(self.head_workspace_size(batch, w1, w2),
                                            dtype=torch.uint8, device=logits.device)
            workspace = self._ws[key]
        st = self._lib.dt_build_tree_head(self.handle, logits.data_ptr(), batch, H.data_ptr(),
                                          ctypes.byref(hd), None if h0 is None else h0.data_ptr(),
                                          T, workspace.data_ptr(), workspace.numel(),
                                          ctypes.byref(out.as_c()), _stream(stream))
        if st != 0:
            _check(st)
        return out

    def set_profiling(self, every: int) -> None:
        """Record stage events on every `every`-th call (0 or False: off)."""
        _check(self._lib.dt_plan_set_profiling(self.handle, int(every)))

    def stage_ms(self) -> dict:
        """Mean kernel durations (ms) over the calls profiled since set_profiling(True)."""
        ms = (ctypes.c_float * 2)()
        _check(self._lib.dt_plan_stage_ms(self.handle, ms))
        return dict(zip(STAGES, list(ms)))

    def set_adaptive_budget(self, c_draft: float = 0.0, c_verify=None) -> None:
        """CaDDTree's stopping rule with cost model (C_d, C_v(0..B)); None: fixed budget."""
        if c_verify is None:
            _check(self._lib.dt_plan_set_adaptive_budget(self.handle, 0.0, None, 0))
            return
        cv = (ctypes.c_float * len(c_verify))(*[float(x) for x in c_verify])
        _check(self._lib.dt_plan_set_adaptive_budget(self.handle, float(c_draft), cv, len(c_verify)))

    def expand_stats(self, n: int):
        """(steps, expanded) per tree of the last profiled call, as int lists."""
        steps = (ctypes.c_int32 * n)()
        expanded = (ctypes.c_int32 * n)()
        _check(self._lib.dt_plan_expand_stats(self.handle, steps, expanded, n))
        return list(steps), list(expanded)

    def close(self) -> None:
        if getattr(self, "handle", None):
            self._lib.dt_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def build_tree(marginal_logits, emb, gru_weights, correction_head, L: int, M: int, B: int,
               T: float, h0=None, max_children: int = 0, norm_mode: int = DT_NORM_TAIL,
               pos_offset: int = 0, scorer: int = DT_SCORER_COND, frontier_width: int = 0) -> Tree:
    """One-shot form of the paper's build_tree(...) -> tree; returns when the trees are built.

    Folds the candidates' embedding rows only where dt_build_tree_once takes the
    shape; otherwise creates and drops a plan (the whole vocabulary folded).
    gru_weights = (w_ih, w_hh, b_ih, b_hh); correction_head = (w_c, b_c).
    """
    import torch
    w_ih, w_hh, b_ih, b_hh = gru_weights
    w_c, b_c = correction_head
    lib = load()
    V, d_e = emb.shape
    d_h, batch = w_hh.shape[1], marginal_logits.shape[0]
    wdt, ldt = _dtype_code(emb), _dtype_code(marginal_logits)
    opts = dt_options(max_children, norm_mode, pos_offset, scorer, frontier_width, 0)
    n = ctypes.c_size_t()
    if lib.dt_once_workspace_size(V, d_e, d_h, wdt, L, M, B, ldt, batch, ctypes.byref(opts),
                                  ctypes.byref(n)) == 0:
        stream = torch.cuda.current_stream()
        default = torch.cuda.default_stream()
        if stream != default:
            stream.wait_stream(default)   # (weights just written there)
        out = Tree.empty(batch, B, marginal_logits.device)
        ws = torch.empty(n.value, dtype=torch.uint8, device=marginal_logits.device)
        gru = dt_gru(_ptr(w_ih), _ptr(w_hh), _ptr(b_ih), _ptr(b_hh), d_e, d_h)
        head = dt_head(_ptr(w_c), _ptr(b_c))
        _check(lib.dt_build_tree_once(_ptr(emb), V, d_e, ctypes.byref(gru), ctypes.byref(head), wdt, L, M, B,
                                      ldt, _ptr(marginal_logits), batch, _ptr(h0), T, ctypes.byref(opts),
                                      ws.data_ptr(), n.value, ctypes.byref(out.as_c()), _stream(stream)))
        stream.synchronize()
        return out
    plan = Plan(emb, w_ih, w_hh, b_ih, b_hh, w_c, b_c, L=L, M=M, B=B,
                logits_dtype=_dtype_code(marginal_logits), max_batch=marginal_logits.shape[0],
                max_children=max_children, norm_mode=norm_mode, pos_offset=pos_offset,
                scorer=scorer, frontier_width=frontier_width)
    try:
        return plan.build_tree(marginal_logits, T, h0)
    finally:
        torch.cuda.current_stream().synchronize()
        plan.close()


def scan_topm(logits, M: int, T: float, stream=None):
    """dt_scan_topm over a [rows, V] tensor: (ids, vals, tail_lse, row_flags)."""
    import torch
    lib = load()
    rows, V = logits.shape
    n = ctypes.c_size_t()
    _check(lib.dt_scan_workspace_size(rows, V, M, ctypes.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device=logits.device)
    ids = torch.empty(rows, M, dtype=torch.int32, device=logits.device)
    vals = torch.empty(rows, M, dtype=torch.float32, device=logits.device)
    tail = torch.empty(rows, dtype=torch.float32, device=logits.device)
    flags = torch.empty(rows, dtype=torch.int32, device=logits.device)
    _check(lib.dt_scan_topm(_ptr(logits), rows, V, _dtype_code(logits), M, ctypes.c_float(T),
                            _ptr(ids), _ptr(vals), _ptr(tail), _ptr(flags), _ptr(ws), n.value,
                            _stream(stream)))
    return ids, vals, tail, flags


# ---- verification: the paged cache, attention over it, the commit of a tree ----------------
# Calls here are short (a kernel of a few us), so their own work is kept small: one lookup of the
# raw stream, C structures that are filled anew rather than made, no checks that the C side makes.

def _want(t, name, shape, dtype, device):
    """A contiguous tensor of this shape and dtype on a device (its index), as the C ABI takes it."""
    if t.dtype != dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: want a contiguous {dtype} tensor of shape {shape} on cuda:{device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _raw_stream(torch, device: int, stream, what: str):
    """The handle of `stream` (None: torch's current one) for a call on a device, which has to be the current one."""
    if device < 0:
        raise ValueError(f"{what} not on a GPU")
    if torch._C._cuda_getDevice() != device:
        raise ValueError(f"{what} on device {device}, which is not the current one")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device) or None
    if stream.device_index != device:
        raise ValueError(f"{what} on device {device}, the stream on device {stream.device_index}")
    return stream.cuda_stream or None


def _empty(torch, shape, dtype, device, stream):
    """A tensor written on `stream` (None: torch's current one) and read on torch's current stream: allocated on
    the first, so that what its memory held before is not still in use, and kept until the second has passed."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _capturing(torch, stream) -> bool:
    """Whether calls on `stream` (None: torch's current one) go into a graph."""
    if stream is None:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


def _keep(stream, *tensors):
    """Tensors of other streams stay allocated until a call on `stream` has used them."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


class Chunk:
    """dt_chunk: the new tokens of a batch of sequences and where they lie in a cache.

    starts [batch + 1], lens [batch] and table [batch, width]: int32 tensors on the cache's device, read when
    the kernels run, so a program may go on changing their contents in place; max_chunk and max_len
    bound the chunks and the lengths they will hold (attention is cut up for max_len tokens: a bound far
    above the lengths is right but slower).
    """

    def __init__(self, starts, lens, table, max_chunk: int, max_len: int):
        import torch
        batch, width = table.shape
        self.device = table.get_device()
        if self.device < 0:
            raise ValueError(f"table: want a tensor on a GPU, got one on {table.device}")
        self.starts = _want(starts, "starts", (batch + 1,), torch.int32, self.device)
        self.lens = _want(lens, "lens", (batch,), torch.int32, self.device)
        self.table = _want(table, "table", (batch, width), torch.int32, self.device)
        self.tensors = starts, lens, table
        self.batch, self.max_chunk, self.max_len = batch, max_chunk, max_len
        self.sizes = (batch, max_chunk, max_len, width)
        self._pointers = starts.data_ptr(), lens.data_ptr(), table.data_ptr()
        self._views = {}

    def as_c(self, rows: int):
        """The dt_chunk of a call with so many rows (by reference): one for each number of rows, not written to
        again, so calls of several host threads may share a Chunk."""
        ref = self._views.get(rows)
        if ref is None:
            if len(self._views) >= 64:   # (a call that holds one keeps it alive)
                self._views = {}
            batch, max_chunk, max_len, width = self.sizes
            ref = self._views[rows] = ctypes.byref(dt_chunk(batch, rows, max_chunk, max_len, width, *self._pointers))
        return ref


@dataclasses.dataclass
class Accepted:
    """dt_tree_accept's results (device tensors)."""
    path: "torch.Tensor"        # [b, B] int32 accepted nodes, then -1
    n_accepted: "torch.Tensor"  # [b] int32
    next_token: "torch.Tensor"  # [b] int32 the target's token after the path


class _Arguments(threading.local):
    """C structures of the functions below, filled anew by every call, and sampling's workspaces: one set for each
    host thread, as threads may call on the same stream."""

    def __init__(self):
        self.rows = [dt_rows() for _ in range(4)]
        self.rotary, self.sampling = dt_rotary(), dt_sampling()
        self.spaces = {}   # a workspace of each stream
        self.refs = [ctypes.byref(x) for x in (*self.rows, self.rotary, self.sampling)]


_arguments = _Arguments()


def _fill_rotary(c: dt_rotary, torch, positions, inv_freq, q_weight, k_weight, eps, interleaved, rows, dim, dtype,
                 device) -> None:
    """The dt_rotary of a call."""
    c.positions = _want(positions, "positions", (rows,), torch.int32, device).data_ptr()
    pairs = inv_freq.numel()
    c.inv_freq, c.pairs = _want(inv_freq, "inv_freq", (pairs,), torch.float32, device).data_ptr(), pairs
    c.q_weight = None if q_weight is None else _want(q_weight, "q_weight", (dim,), dtype, device).data_ptr()
    c.k_weight = None if k_weight is None else _want(k_weight, "k_weight", (dim,), dtype, device).data_ptr()
    c.eps, c.interleaved = eps, interleaved


class Cache:
    """dt_cache: keys and values of `layers` layers in pages, in the kernels' own order.

    dtype: torch.float32, torch.bfloat16 or torch.float8_e4m3fn (bf16 data with one power-of-two
    scale for each token and head).  Calls run on torch's current stream of the cache's device
    unless one is given (which has to wait for what made its inputs, and be waited for, as any);
    workspaces are kept for each stream.  A captured call has a workspace from its graph's memory
    (torch.cuda.graph's), which no other call is given while the graph lives: replays and other calls
    may overlap.  A stream that is captured by other means needs `workspace`.
    A Cache is used by one host thread at a time, with its device as the current one.
    """

    def __init__(self, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype, layers: int = 1,
                 device="cuda"):
        import torch
        codes = {torch.float32: DT_F32, torch.bfloat16: DT_BF16, torch.float8_e4m3fn: DT_F8}
        if dtype not in codes:
            raise TypeError(f"unsupported dtype {dtype}")
        self._lib, self._torch = load(), torch
        self.pages, self.page_size, self.kv_heads, self.head_dim, self.layers = (pages, page_size, kv_heads,
                                                                                head_dim, layers)
        self.dtype = dtype
        self.data_dtype, self._data_bytes = (torch.float32, 4) if dtype == torch.float32 else (torch.bfloat16, 2)
        c = dt_cache(None, layers, pages, page_size, kv_heads, head_dim, codes[dtype])
        n = ctypes.c_size_t()
        _check(self._lib.dt_cache_size(ctypes.byref(c), ctypes.byref(n)))
        self.storage = torch.empty(n.value, dtype=torch.uint8, device=device)
        c.data = self.storage.data_ptr()
        self._c, self._ref = c, ctypes.byref(c)
        self._at = self.storage.device
        self._device = self._at.index
        self._a, self._b, self._o = dt_rows(), dt_rows(), dt_attend_options()   # a call's arguments
        self._aref, self._bref, self._oref = (ctypes.byref(x) for x in (self._a, self._b, self._o))
        self._scale = head_dim ** -0.5
        self._sizes = {}   # workspace bytes of a shape
        self._ws = {}      # a workspace of each stream

    def _stream(self, stream):
        return _raw_stream(self._torch, self._device, stream, "the cache is")

    def _chunk(self, chunk: Chunk, rows: int):
        """The dt_chunk of a call with so many rows (by reference)."""
        if chunk.device != self._device:
            raise ValueError(f"the chunk's tensors are on device {chunk.device}, the cache is on {self._device}")
        return chunk.as_c(rows)

    def _rows(self, c: dt_rows, t, name: str, heads: Optional[int] = None) -> int:
        """Fill c from a tensor [rows, heads, head_dim]; its rows."""
        shape, stride = t.shape, t.stride()
        if t.dtype != self.data_dtype or len(shape) != 3 or shape[2] != self.head_dim or \
                t.get_device() != self._device or (heads is not None and shape[1] != heads):
            raise ValueError(f"{name}: want a {self.data_dtype} tensor [rows, {heads or 'heads'}, {self.head_dim}] "
                             f"on {self._at}, got {t.dtype} {tuple(shape)} on {t.device}")
        if stride[2] != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous (stride {stride[2]})")
        c.data = t.data_ptr()
        c.row_stride, c.head_stride = stride[0], stride[1]
        return shape[0]

    def _kv(self, k, v) -> int:
        rows = self._rows(self._a, k, "k", self.kv_heads)
        if self._rows(self._b, v, "v", self.kv_heads) != rows:
            raise ValueError(f"k and v have {rows} and {v.shape[0]} rows")
        return rows

    def append(self, chunk: Chunk, k, v, layer: int = 0, stream=None) -> None:
        """dt_cache_append: the chunk's keys and values [rows, kv_heads, head_dim] into a layer."""
        rows = self._kv(k, v)
        st = self._lib.dt_cache_append(self._ref, layer, self._chunk(chunk, rows), self._aref, self._bref,
                                       self._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.storage, k, v, *chunk.tensors)

    def append_rotated(self, chunk: Chunk, q, k, v, positions, inv_freq, q_weight=None, k_weight=None,
                       eps: float = 1e-6, interleaved: bool = False, layer: int = 0, out=None, stream=None):
        """dt_cache_append_rotated: rotate and append in one: the chunk's keys, normed and rotated, and values
        into a layer; its queries [rows, heads, head_dim], normed and rotated, as the result (`out` may be q).

        positions, inv_freq, the weights, eps and interleaved are rotate's.  Rows of no chunk are left as they are.
        """
        torch = self._torch
        rows = self._kv(k, v)
        (x, y, _, _), refs = _arguments.rows, _arguments.refs
        if self._rows(x, q, "q") != rows:
            raise ValueError(f"q and k have {q.shape[0]} and {rows} rows")
        heads, dim = q.shape[1], self.head_dim
        if out is None:
            out = _empty(torch, (rows, heads, dim), self.data_dtype, self._at, stream)
            y.data, y.row_stride, y.head_stride = out.data_ptr(), heads * dim, dim
        elif self._rows(y, out, "out", heads) != rows:
            raise ValueError(f"q and out have {rows} and {out.shape[0]} rows")
        _fill_rotary(_arguments.rotary, torch, positions, inv_freq, q_weight, k_weight, eps, interleaved, rows, dim,
                     self.data_dtype, self._device)
        st = self._lib.dt_cache_append_rotated(self._ref, layer, self._chunk(chunk, rows), heads, refs[0], self._aref,
                                               self._bref, refs[4], refs[1], self._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.storage, q, k, v, out, positions, inv_freq, q_weight, k_weight, *chunk.tensors)
        return out

    def read(self, chunk: Chunk, rows: Optional[int] = None, layer: int = 0, out=None, stream=None):
        """dt_cache_read: the chunk's keys and values as (k, v) [rows, kv_heads, head_dim].

        rows: rows of the tensors made (starts' last); out = (k, v) takes given ones instead.
        Rows that belong to no chunk are left as they are.
        """
        if out is None:
            if rows is None:
                raise ValueError("read needs the number of rows, or out")
            both = _empty(self._torch, (2, rows, self.kv_heads, self.head_dim), self.data_dtype, self._at, stream)
            a, b = self._a, self._b
            a.data = at = both.data_ptr()
            a.head_stride = b.head_stride = self.head_dim
            a.row_stride = b.row_stride = row = self.kv_heads * self.head_dim
            b.data = at + rows * row * self._data_bytes
        else:
            rows = self._kv(*out)
        st = self._lib.dt_cache_read(self._ref, layer, self._chunk(chunk, rows), self._aref, self._bref,
                                     self._stream(stream))
        if st != 0:
            _check(st)
        if out is None:
            out = both.unbind(0)
        if stream is not None:
            _keep(stream, self.storage, *out, *chunk.tensors)
        return out

    def workspace_size(self, chunk: Chunk, rows: int, heads: int, opts: dt_attend_options) -> int:
        return self._workspace_size(chunk, rows, heads, opts, opts.window, opts.sinks, opts.tree_nodes)

    def _workspace_size(self, chunk: Chunk, rows: int, heads: int, opts: dt_attend_options, window, sinks, nodes) -> int:
        key = (chunk.sizes, rows, heads, window, sinks, nodes)
        n = self._sizes.get(key)
        if n is None:
            if len(self._sizes) >= 4096:   # (shapes of a long-running program)
                self._sizes.clear()
            b = ctypes.c_size_t()
            _check(self._lib.dt_attend_workspace_size(self._ref, chunk.as_c(rows), heads, ctypes.byref(opts),
                                                      ctypes.byref(b)))
            n = self._sizes[key] = b.value
        return n

    def _workspace(self, n: int, raw, stream):
        """The stream's workspace, grown to n bytes: allocated on that stream, where calls follow one another, so an
        outgrown one may go.  A graph's calls come again after that: what they use is the graph's, not the stream's."""
        if _capturing(self._torch, stream):
            return _empty(self._torch, (n,), self._torch.uint8, self._at, stream)
        ws = self._ws.get(raw)
        if ws is None or ws.numel() < n:
            ws = self._ws[raw] = _empty(self._torch, (n,), self._torch.uint8, self._at, stream)
        return ws

    def attend(self, chunk: Chunk, q, scale: Optional[float] = None, layer: int = 0, window: int = 0,
               sinks: int = 0, mask=None, depth=None, out=None, workspace=None, stream=None):
        """dt_cache_attend: attention of the chunk's queries q [rows, heads, head_dim] over a layer.

        scale: default head_dim ** -0.5; window (0: none) with `sinks` first tokens that stay visible;
        mask [batch, N, N] uint8 (Tree.mask): the last N rows of every chunk are a tree's nodes, depth
        [batch, N] (Tree.depth) their depths, needed with a window.
        """
        rows, heads, d = self._rows(self._a, q, "q"), q.shape[1], self.head_dim
        if out is None:
            if stream is None and q.is_contiguous():
                out = self._torch.empty_like(q)
            else:
                out = _empty(self._torch, (rows, heads, d), self.data_dtype, self._at, stream)
            b = self._b
            b.data, b.row_stride, b.head_stride = out.data_ptr(), heads * d, d
        elif self._rows(self._b, out, "out", heads) != rows:
            raise ValueError(f"q and out have {rows} and {out.shape[0]} rows")
        o = self._o
        o.scale = self._scale if scale is None else scale
        o.window, o.sinks, nodes = window, sinks, 0
        o.mask = o.depth = None
        if mask is not None:
            nodes = mask.shape[-1]
            o.mask = _want(mask, "mask", (chunk.batch, nodes, nodes), self._torch.uint8,
                           self._device).data_ptr()
            if depth is not None:
                o.depth = _want(depth, "depth", (chunk.batch, nodes), self._torch.int32,
                                self._device).data_ptr()
        o.tree_nodes = nodes
        s = self._stream(stream)
        if workspace is None:
            n = self._workspace_size(chunk, rows, heads, o, window, sinks, nodes)
            if n:
                workspace = self._workspace(n, s, stream)
        elif workspace.get_device() != self._device or not workspace.is_contiguous():
            raise ValueError(f"workspace: want a contiguous tensor on {self._at}, got one on {workspace.device}")
        ws, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())
        st = self._lib.dt_cache_attend(self._ref, layer, self._chunk(chunk, rows), heads, self._aref, self._bref,
                                       self._oref, ws, size, s)
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.storage, q, out, mask, depth, workspace, *chunk.tensors)
        return out

    def copy_pages(self, source, to, stream=None) -> None:
        """dt_cache_copy_pages: pages `to` [n] become copies of pages `source` [n] (int32) in every layer."""
        n, i32 = source.numel(), self._torch.int32
        _want(source, "source", (n,), i32, self._device)
        _want(to, "to", (n,), i32, self._device)
        st = self._lib.dt_cache_copy_pages(self._ref, source.data_ptr(), to.data_ptr(), n, self._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.storage, source, to)

    def commit(self, chunk: Chunk, path, n_accepted, stream=None) -> None:
        """dt_cache_commit: the rows of the accepted nodes (Accepted.path, .n_accepted) moved together, in
        every layer; the nodes are the last path.shape[1] rows of each chunk."""
        i32 = self._torch.int32
        n = path.shape[1]
        _want(path, "path", (chunk.batch, n), i32, self._device)
        _want(n_accepted, "n_accepted", (chunk.batch,), i32, self._device)
        every = min(chunk.batch * chunk.max_chunk, 2 ** 31 - 1)   # (no tensor of rows here: starts' bound)
        st = self._lib.dt_cache_commit(self._ref, self._chunk(chunk, every), n, path.data_ptr(), n_accepted.data_ptr(),
                                       self._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.storage, path, n_accepted, *chunk.tensors)


class Pages:
    """dt_pages: which pages of a cache the sequences of a batch hold.

    `lens` [batch] are the sequences' tokens, set by the program (in place); fit() then gives and takes pages,
    fork() makes sequences copies of others, compact() moves the pages in use together.  `table` and `lens` may be a
    Chunk's.  All are int32 tensors on the cache's device, views of `state`, which holds the whole books (to be saved and
    copied back): missing [1], uses [pages], held [batch], lens, table [batch, width].
    missing: pages that the last call lacked; it then grew and forked nothing.
    A sequence that is cut back into a page that others hold is forked into another place before it is appended to.
    Calls run on torch's current stream of the cache's device unless one is given; they use one workspace, so calls of one
    Pages (captured ones too) must not overlap, as they change the same books.
    """

    def __init__(self, cache: Cache, batch: int, width: int):
        torch = cache._torch
        self.cache, self.batch, self.width = cache, batch, width
        c = dt_pages(cache.pages, cache.page_size, batch, width)
        n = ctypes.c_size_t()
        _check(cache._lib.dt_pages_workspace_size(ctypes.byref(c), ctypes.byref(n)))
        sizes = 1, cache.pages, batch, batch, batch * width
        self.state = torch.zeros(sum(sizes), dtype=torch.int32, device=cache._at)
        self.missing, self.uses, self.held, self.lens, table = self.state.split(sizes)
        self.table = table.view(batch, width)
        self.table.fill_(-1)
        self._ws = torch.empty(n.value, dtype=torch.uint8, device=cache._at)
        c.uses, c.held, c.lens, c.table, c.missing = (t.data_ptr() for t in (self.uses, self.held, self.lens, self.table,
                                                                             self.missing))
        self._c, self._ref, self._bytes = c, ctypes.byref(c), n.value

    def fit(self, stream=None) -> None:
        """dt_pages_fit: every sequence holds the pages of its lens, no more and, if all can be served, no fewer."""
        cache = self.cache
        st = cache._lib.dt_pages_fit(self._ref, self._ws.data_ptr(), self._bytes, cache._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.state, self._ws)

    def fork(self, source, stream=None) -> None:
        """dt_pages_fork: sequence b becomes a copy of sequence source[b] ([batch] int32), for all b at once."""
        cache = self.cache
        _want(source, "source", (self.batch,), cache._torch.int32, cache._device)
        st = cache._lib.dt_pages_fork(self._ref, cache._ref, source.data_ptr(), self._ws.data_ptr(), self._bytes,
                                      cache._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.state, self._ws, cache.storage, source)

    def compact(self, stream=None) -> None:
        """dt_pages_compact: the n pages in use become the cache's first n."""
        cache = self.cache
        st = cache._lib.dt_pages_compact(self._ref, cache._ref, self._ws.data_ptr(), self._bytes, cache._stream(stream))
        if st != 0:
            _check(st)
        if stream is not None:
            _keep(stream, self.state, self._ws, cache.storage)


def _fill_rows(c: dt_rows, t, name: str, device: int, dtype, rows=None, heads=None, dim=None) -> None:
    """The dt_rows of a tensor [rows, heads, dim] (None: any)."""
    shape, stride = t.shape, t.stride()
    if t.dtype != dtype or len(shape) != 3 or t.get_device() != device or (rows is not None and shape[0] != rows) or \
            (heads is not None and shape[1] != heads) or (dim is not None and shape[2] != dim):
        want = [x or n for x, n in ((rows, "rows"), (heads, "heads"), (dim, "dim"))]
        raise ValueError(f"{name}: want a {dtype} tensor [{want[0]}, {want[1]}, {want[2]}] on cuda:{device}, "
                         f"got {t.dtype} {tuple(shape)} on {t.device}")
    if stride[2] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous (stride {stride[2]})")
    c.data, c.row_stride, c.head_stride = t.data_ptr(), stride[0], stride[1]


def rotate(q, k, positions, inv_freq, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
           out=None, stream=None):
    """dt_rotate: queries [rows, heads, D] and keys [rows, kv_heads, D] (None: queries alone), float32 or bfloat16,
    normed (where a weight [D] of their dtype is given) and rotated by position; (q, k).

    positions [rows] int32 (Tree.position_ids, for a tree's nodes); inv_freq [pairs] float32, pairs a multiple of 8
    and at most D / 2: element j is paired with j + pairs, or with interleaved 2 j with 2 j + 1.
    out = (q, k) takes given tensors, which may be the inputs themselves.  Runs on torch's current
    stream of the tensors' device (the current one) unless one is given.
    """
    import torch
    device, dtype, code = q.get_device(), q.dtype, _dtype_code(q)
    s = _raw_stream(torch, device, stream, "q is")
    (x, y, a, b), refs = _arguments.rows, _arguments.refs
    _fill_rows(x, q, "q", device, dtype)
    rows, heads, dim = q.shape
    kv = 0
    if k is not None:
        kv = k.shape[1]
        _fill_rows(y, k, "k", device, dtype, rows, dim=dim)
    if out is None:
        # (one allocation, parted as the calls for cached rows do)
        n = rows * heads * dim
        both = _empty(torch, (n + rows * kv * dim,), dtype, q.device, stream)
        out = both.as_strided((rows, heads, dim), (heads * dim, dim, 1)), \
            None if k is None else both.as_strided((rows, kv, dim), (kv * dim, dim, 1), n)
        a.data = at = both.data_ptr()
        a.row_stride, a.head_stride = heads * dim, dim
        b.data, b.row_stride, b.head_stride = at + n * both.element_size(), kv * dim, dim
    else:
        _fill_rows(a, out[0], "out", device, dtype, rows, heads, dim)
        if k is not None:
            _fill_rows(b, out[1], "out", device, dtype, rows, kv, dim)
    _fill_rotary(_arguments.rotary, torch, positions, inv_freq, q_weight, k_weight, eps, interleaved, rows, dim, dtype, device)
    st = load().dt_rotate(refs[0], heads, None if k is None else refs[1], kv, rows, dim, code, refs[4], refs[2],
                          None if k is None else refs[3], s)
    if st != 0:
        _check(st)
    if stream is not None:
        _keep(stream, q, k, positions, inv_freq, q_weight, k_weight, *out)
    return out


_sample_bytes = {}   # of a workspace for (rows, V)
_SPACE_BYTES, _SPACES = 32 << 20, 8   # workspaces that a host thread keeps: their largest size, how many


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, logprobs=False, workspace=None,
           stream=None):
    """dt_sample: a token of each row of logits [..., V] (float32 or bfloat16) by random numbers u [...] float32 in
    [0, 1): int32 tokens [...], with a batch of trees' roots and nodes [b, B + 1, V] accept_tree's target.

    temperature (0: the largest logit), top_k (0: off), top_p (1: off) and min_p (0: off): a number for every row, or a
    tensor of u's shape (float32; top_k int32).  logprobs=True also returns the tokens' float32 log-probabilities
    within what is kept: (tokens, logprobs).  out takes given tensors: tokens, or with logprobs both.  The last
    dimension is contiguous, the others lie at one stride (padded rows do).  Runs on torch's current
    stream of the tensors' device (the current one) unless one is given.
    A host thread keeps the workspaces of a few streams, up to 32 MiB each; larger ones (from about 1,100 rows of a large
    vocabulary on) are allocated by each call, unless `workspace` gives one (of dt_sample_workspace_size's bytes).
    """
    import torch
    lib = load()
    device, shape = logits.get_device(), logits.shape[:-1]
    code = _dtype_code(logits)
    s = _raw_stream(torch, device, stream, "logits are")
    if len(shape) != 1:
        try:
            logits = logits.view(-1, logits.shape[-1])
        except RuntimeError as e:
            raise ValueError(f"logits: the rows do not lie at one stride ({logits.stride()})") from e
    rows, V = logits.shape
    if logits.stride(1) != 1 and V > 1:
        raise ValueError(f"logits: the last dimension must be contiguous (stride {logits.stride(1)})")
    f32, i32 = torch.float32, torch.int32
    _want(u, "u", shape, f32, device)
    how, kept = _arguments.sampling, []
    for name, names, x, dtype in (("temperature", "temperatures", temperature, f32), ("top_k", "top_ks", top_k, i32),
                                  ("top_p", "top_ps", top_p, f32), ("min_p", "min_ps", min_p, f32)):
        if isinstance(x, torch.Tensor):
            setattr(how, names, _want(x, name, shape, dtype, device).data_ptr())
            kept.append(x)
        else:
            setattr(how, names, None)
            # (top_k: a C int drops the bits above its 32; V is as good as more, and -1 is refused as less is)
            setattr(how, name, max(-1, min(operator.index(x), V)) if name == "top_k" else x)
    if workspace is None:
        n = _sample_bytes.get((rows, V))
        if n is None:
            size = ctypes.c_size_t()
            _check(lib.dt_sample_workspace_size(rows, V, ctypes.byref(size)))
            if len(_sample_bytes) >= 4096:   # (shapes of a long-running program)
                _sample_bytes.clear()
            n = _sample_bytes[(rows, V)] = size.value
        # (kept for the stream, where calls follow one another; a graph's calls come again after that, and have their own.
        # Kept up to a bound: a call of more rows takes far longer than an allocation)
        spaces, at = _arguments.spaces, (device, s)
        workspace = None if _capturing(torch, stream) else spaces.get(at)
        if workspace is None or workspace.numel() < n:
            workspace = _empty(torch, (n,), torch.uint8, logits.device, stream)
            if n <= _SPACE_BYTES and not _capturing(torch, stream):
                if len(spaces) >= _SPACES:
                    spaces.clear()
                spaces[at] = workspace
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError(f"workspace: want a contiguous tensor on cuda:{device}, got one on {workspace.device}")
    if out is None:
        tokens = _empty(torch, shape, i32, logits.device, stream)
        probs = _empty(torch, shape, f32, logits.device, stream) if logprobs else None
    else:
        tokens, probs = out if logprobs else (out, None)
        _want(tokens, "out", shape, i32, device)
        if logprobs:
            _want(probs, "out", shape, f32, device)
    st = lib.dt_sample(logits.data_ptr(), logits.stride(0), rows, V, code, u.data_ptr(), _arguments.refs[5], tokens.data_ptr(),
                       None if probs is None else probs.data_ptr(), workspace.data_ptr(),
                       workspace.numel() * workspace.element_size(), s)
    if st != 0:
        _check(st)
    if stream is not None:
        _keep(stream, logits, u, tokens, probs, workspace, *kept)
    return (tokens, probs) if logprobs else tokens


def accept_tree(tree: Tree, target, out: Optional[Accepted] = None, stream=None) -> Accepted:
    """dt_tree_accept: the longest path of each tree that the target agrees with.

    target [b, B + 1] int32: the target's token at the root and at every node.  Runs on torch's current stream
    of the tensors' device (the current one) unless one is given; out: results to write instead of new ones.
    """
    import torch
    b, B = tree.tokens.shape
    i32, device = torch.int32, target.get_device()
    s = _raw_stream(torch, device, stream, "target is")
    _want(target, "target", (b, B + 1), i32, device)
    if tree.__dict__.get("_device") != device:   # (looked at once, as its C view is made once)
        for name, shape in (("tokens", (b, B)), ("parents", (b, B)), ("n_nodes", (b,))):
            _want(getattr(tree, name), name, shape, i32, device)
        tree.__dict__["_device"] = device
    if out is None:
        path, n, token = _empty(torch, (b * (B + 2),), i32, target.device, stream).split_with_sizes((b * B, b, b))
        out = Accepted(path.view(b, B), n, token)
    else:
        for name, shape in (("path", (b, B)), ("n_accepted", (b,)), ("next_token", (b,))):
            _want(getattr(out, name), name, shape, i32, device)
    st = load().dt_tree_accept(ctypes.byref(tree.as_c()), b, B, target.data_ptr(), out.path.data_ptr(),
                               out.n_accepted.data_ptr(), out.next_token.data_ptr(), s)
    if st != 0:
        _check(st)
    if stream is not None:
        _keep(stream, tree.tokens, tree.parents, tree.n_nodes, target, out.path, out.n_accepted, out.next_token)
    return out
