"""Python binding of libtod's C ABI (argument marshalling only).

Every function here has the name of the C entry point it calls and does no
arithmetic of its own: torch supplies device memory and the current HIP
stream; all work runs in the library's HIP kernels.  Importing this module
raises ImportError if ``libtod.so`` has not been built (there is no CPU or
PyTorch fallback).
"""
from __future__ import annotations

import ctypes
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtod.so")

TOD_OK = 0
TOD_ERR_INVALID_ARG = 1
TOD_ERR_NONFINITE = 2
TOD_ERR_WORKSPACE = 3
TOD_ERR_UNSUPPORTED = 4
TOD_ERR_HIP = 5
TOD_ERR_INTERNAL = 6
TOD_ERR_CAPACITY = 7

PREC_AUTO, PREC_FP32, PREC_FP16, PREC_BF16 = 0, 1, 2, 3
PRECISIONS = {"auto": PREC_AUTO, "fp32": PREC_FP32, "fp16": PREC_FP16, "bf16": PREC_BF16}
PRECISION_NAMES = {v: k for k, v in PRECISIONS.items()}
SCORES = {"kth": 0, "largest": 0, "mean": 1, "median": 2, "sum": 3}

SYMBOLS = ("tod_default_options", "tod_workspace_size", "tod_knn", "tod_knn_noalloc",
           "tod_knn_score", "tod_lof", "tod_lof_ties_workspace_size", "tod_lof_ties",
           "tod_knn_decision", "tod_knn_classify", "tod_abod", "tod_cof", "tod_nwr_workspace_size",
           "tod_nwr", "tod_loci_workspace_size", "tod_loci",
           "tod_plan", "tod_plan_workspace", "tod_page_map", "tod_page_write",
           "tod_default_attn", "tod_attn_workspace_size", "tod_attn_prompt", "tod_attn_paged",
           "tod_default_append", "tod_page_append", "tod_status_string", "tod_last_error")
# Those of a 4-bit cache.
SYMBOLS4 = ("tod_page_append4", "tod_page_read4", "tod_attn_paged4_workspace_size",
            "tod_attn_paged4")


class tod_options(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("precision", ctypes.c_int32),
        ("exclude_self", ctypes.c_int32),
        ("shortlist", ctypes.c_int32),
        ("query_block", ctypes.c_int64),
        ("ref_splits", ctypes.c_int32),
        ("margin_scale", ctypes.c_float),
        ("force_fallback", ctypes.c_int32),
        ("no_recheck", ctypes.c_int32),
        ("reorder", ctypes.c_int32),
        ("score", ctypes.c_int32),
        ("tail_parts", ctypes.c_int32),
    ]


class tod_stats(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("precision", ctypes.c_int32),
        ("kprime", ctypes.c_int32),
        ("ref_splits", ctypes.c_int32),
        ("query_block", ctypes.c_int64),
        ("blocks", ctypes.c_int64),
        ("rows_certified", ctypes.c_int64),
        ("rows_fallback", ctypes.c_int64),
        ("tile_launches", ctypes.c_int64),
        ("ms_prep", ctypes.c_float),
        ("ms_tile", ctypes.c_float),
        ("ms_recheck", ctypes.c_float),
        ("ms_fallback", ctypes.c_float),
        ("ms_score", ctypes.c_float),
        ("ms_total", ctypes.c_float),
        ("reordered", ctypes.c_int32),
        ("pairs_candidate", ctypes.c_int64),
        ("pairs_uncertain", ctypes.c_int64),
        ("pairs_in_range", ctypes.c_int64),
        ("tail_parts", ctypes.c_int32),
        ("tail_rows", ctypes.c_int64),
        ("list_runs", ctypes.c_int32),
        ("pruned_kind", ctypes.c_int32),
        ("pruned_blocks", ctypes.c_int64),
        ("pairs_scanned", ctypes.c_int64),
    ]

    def as_dict(self) -> dict:
        out = {name: getattr(self, name) for name, _ in self._fields_ if name != "struct_size"}
        out["precision"] = PRECISION_NAMES.get(self.precision, self.precision)
        return out


class tod_attn(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("precision", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("dim", ctypes.c_int32),
        ("causal", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("q_row", ctypes.c_int64),
        ("q_head", ctypes.c_int64),
        ("k_row", ctypes.c_int64),
        ("k_head", ctypes.c_int64),
        ("v_row", ctypes.c_int64),
        ("v_head", ctypes.c_int64),
    ]


class tod_append(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("precision", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("dim", ctypes.c_int32),
        ("rotary", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("q_row", ctypes.c_int64),
        ("q_head", ctypes.c_int64),
        ("k_row", ctypes.c_int64),
        ("k_head", ctypes.c_int64),
        ("v_row", ctypes.c_int64),
        ("v_head", ctypes.c_int64),
    ]


class tod_cache4(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("page_rows", ctypes.c_int32),
        ("n_pages", ctypes.c_int64),
        ("k_codes", ctypes.c_void_p),
        ("v_codes", ctypes.c_void_p),
        ("k_scales", ctypes.c_void_p),
        ("v_scales", ctypes.c_void_p),
    ]


class TodError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__("%s failed: %s (%s)" % (where, status_string(status), detail))


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libtod.so is not built (expected at %s); run __graft_entry__.build() or "
            "python paper_2110_14007_amd/build.py" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    opt_p, st_p = ctypes.POINTER(tod_options), ctypes.POINTER(tod_stats)
    lib.tod_default_options.argtypes = [opt_p]
    lib.tod_default_options.restype = None
    lib.tod_workspace_size.argtypes = [i64, i64, i64, i32, i32, opt_p]
    lib.tod_workspace_size.restype = sz
    lib.tod_knn.argtypes = [vp, i64, vp, i64, i64, i32, opt_p, vp, sz, vp, vp, vp, st_p]
    lib.tod_knn.restype = ctypes.c_int
    lib.tod_knn_noalloc.argtypes = [vp, i64, vp, i64, i64, i32, opt_p, vp, vp, vp, st_p]
    lib.tod_knn_noalloc.restype = ctypes.c_int
    lib.tod_knn_score.argtypes = [vp, i64, i64, i32, opt_p, vp, sz, vp, vp, vp, vp, st_p]
    lib.tod_knn_score.restype = ctypes.c_int
    lib.tod_lof.argtypes = [vp, i64, i64, i32, opt_p, vp, sz, vp, vp, vp, vp, vp, st_p]
    lib.tod_lof.restype = ctypes.c_int
    lib.tod_lof_ties_workspace_size.argtypes = [i64, i64, i32, i64, opt_p]
    lib.tod_lof_ties_workspace_size.restype = sz
    lib.tod_lof_ties.argtypes = [vp, i64, i64, i32, i64, opt_p, vp, sz, vp, vp, vp, st_p]
    lib.tod_lof_ties.restype = ctypes.c_int
    lib.tod_knn_decision.argtypes = [vp, i64, vp, i64, i64, i32, opt_p, vp, sz, vp, vp, vp, vp,
                                      st_p]
    lib.tod_knn_decision.restype = ctypes.c_int
    lib.tod_knn_classify.argtypes = [vp, i64, vp, i64, i64, i32, vp, i32, opt_p, vp, sz, vp, vp,
                                     st_p]
    lib.tod_knn_classify.restype = ctypes.c_int
    lib.tod_abod.argtypes = [vp, i64, i64, i32, opt_p, vp, sz, vp, vp, vp, vp, st_p]
    lib.tod_cof.argtypes = [vp, i64, i64, i32, opt_p, vp, sz, vp, vp, vp, vp, vp, st_p]
    lib.tod_cof.restype = ctypes.c_int
    lib.tod_abod.restype = ctypes.c_int
    lib.tod_nwr_workspace_size.argtypes = [i64, i64, i64, opt_p]
    lib.tod_nwr_workspace_size.restype = sz
    lib.tod_nwr.argtypes = [vp, i64, vp, i64, i64, ctypes.c_double, opt_p, vp, sz, vp, vp, i64, vp,
                            vp, ctypes.POINTER(i64), st_p]
    lib.tod_nwr.restype = ctypes.c_int
    dbl = ctypes.c_double
    lib.tod_loci_workspace_size.argtypes = [i64, i64, i32, i64, opt_p]
    lib.tod_loci_workspace_size.restype = sz
    lib.tod_loci.argtypes = [vp, i64, i64, ctypes.POINTER(dbl), i32, dbl, i32, dbl, i64, opt_p, vp,
                             sz, vp, vp, vp, vp, vp, vp, vp, st_p]
    lib.tod_loci.restype = ctypes.c_int
    lib.tod_plan.argtypes = [i64, i64, i64, i32, opt_p, st_p]
    lib.tod_plan.restype = ctypes.c_int
    lib.tod_plan_workspace.argtypes = [i64, i64, i64, i32, i32, opt_p, sz, st_p]
    lib.tod_plan_workspace.restype = ctypes.c_int
    at_p = ctypes.POINTER(tod_attn)
    lib.tod_page_map.argtypes = [vp, vp, i64, vp, i64, i32, vp, i64, i64, vp, vp, vp, vp, vp]
    lib.tod_page_map.restype = ctypes.c_int
    lib.tod_page_write.argtypes = [vp, vp, i64, i32, i32, i64, i64, i64, i64, vp, vp, vp, i64, i32,
                                   vp]
    lib.tod_page_write.restype = ctypes.c_int
    lib.tod_default_attn.argtypes = [at_p, i32, i32, i32, i32]
    lib.tod_default_attn.restype = None
    lib.tod_attn_workspace_size.argtypes = [at_p, i64, i64, i64]
    lib.tod_attn_workspace_size.restype = sz
    lib.tod_attn_prompt.argtypes = [at_p, vp, vp, vp, i64, vp, i64, vp, sz, vp, vp, vp]
    lib.tod_attn_prompt.restype = ctypes.c_int
    lib.tod_attn_paged.argtypes = [at_p, vp, vp, vp, i64, i32, vp, i64, vp, vp, i64, i64, i64, vp,
                                   sz, vp, vp, vp]
    lib.tod_attn_paged.restype = ctypes.c_int
    ap_p, c4_p = ctypes.POINTER(tod_append), ctypes.POINTER(tod_cache4)
    lib.tod_default_append.argtypes = [ap_p, i32, i32, i32, i32]
    lib.tod_default_append.restype = None
    lib.tod_page_append.argtypes = [ap_p, vp, vp, vp, i64, vp, vp, vp, vp, vp, i64, i32, vp, vp]
    lib.tod_page_append.restype = ctypes.c_int
    lib.tod_page_append4.argtypes = [ap_p, vp, vp, vp, i64, vp, vp, vp, c4_p, vp, vp]
    lib.tod_page_append4.restype = ctypes.c_int
    lib.tod_page_read4.argtypes = [c4_p, i32, i32, i32, vp, i64, vp, vp, vp]
    lib.tod_page_read4.restype = ctypes.c_int
    lib.tod_attn_paged4_workspace_size.argtypes = [at_p, i64, i64, i64]
    lib.tod_attn_paged4_workspace_size.restype = sz
    lib.tod_attn_paged4.argtypes = [at_p, vp, c4_p, vp, i64, vp, vp, i64, i64, i64, vp, sz, vp, vp,
                                    vp]
    lib.tod_attn_paged4.restype = ctypes.c_int
    lib.tod_status_string.argtypes = [ctypes.c_int]
    lib.tod_status_string.restype = ctypes.c_char_p
    lib.tod_last_error.argtypes = []
    lib.tod_last_error.restype = ctypes.c_char_p
    return lib


_lib = _load()


def status_string(status: int) -> str:
    return _lib.tod_status_string(int(status)).decode()


def last_error() -> str:
    return _lib.tod_last_error().decode()


def options(precision="auto", exclude_self=False, shortlist=0, query_block=0, ref_splits=0,
            margin_scale=1.0, force_fallback=False, no_recheck=False, reorder=0,
            score="kth", tail_parts=0) -> tod_options:
    o = tod_options()
    _lib.tod_default_options(ctypes.byref(o))
    o.precision = PRECISIONS[precision] if isinstance(precision, str) else int(precision)
    o.exclude_self = int(bool(exclude_self))
    o.shortlist = int(shortlist)
    o.query_block = int(query_block)
    o.ref_splits = int(ref_splits)
    o.margin_scale = float(margin_scale)
    o.force_fallback = int(bool(force_fallback))
    o.no_recheck = int(bool(no_recheck))
    o.reorder = int(reorder)
    o.score = SCORES[score] if isinstance(score, str) else int(score)
    o.tail_parts = int(tail_parts)
    return o


def new_stats() -> tod_stats:
    s = tod_stats()
    s.struct_size = ctypes.sizeof(tod_stats)
    return s


def _check(status: int, where: str):
    if status != TOD_OK:
        raise TodError(status, where, last_error())


def tod_workspace_size(nq: int, nr: int, d: int, k: int, mode: int = 0, opts=None) -> int:
    """mode 0: kNN / scores / decision, 1 (or True): LOF, 2: classifier."""
    return int(_lib.tod_workspace_size(int(nq), int(nr), int(d), int(k), int(mode),
                                       ctypes.byref(opts) if opts is not None else None))


def tod_plan_workspace(nq: int, nr: int, d: int, k: int, ws_bytes: int, mode: int = 0,
                       opts=None) -> dict:
    """Plan of a call with a workspace of ws_bytes (host only)."""
    s = new_stats()
    st = _lib.tod_plan_workspace(int(nq), int(nr), int(d), int(k), int(mode),
                                 ctypes.byref(opts) if opts is not None else None,
                                 ctypes.c_size_t(int(ws_bytes)), ctypes.byref(s))
    _check(st, "tod_plan_workspace")
    return {"precision": PRECISION_NAMES[s.precision], "kprime": s.kprime,
            "ref_splits": s.ref_splits, "query_block": s.query_block, "blocks": s.blocks,
            "reordered": s.reordered, "list_runs": s.list_runs, "pruned_kind": s.pruned_kind}


def tod_plan(nq: int, nr: int, d: int, k: int, opts=None) -> dict:
    s = new_stats()
    _check(_lib.tod_plan(int(nq), int(nr), int(d), int(k),
                         ctypes.byref(opts) if opts is not None else None, ctypes.byref(s)),
           "tod_plan")
    return {"precision": PRECISION_NAMES[s.precision], "kprime": s.kprime,
            "ref_splits": s.ref_splits, "query_block": s.query_block, "blocks": s.blocks,
            "reordered": bool(s.reordered), "list_runs": s.list_runs,
            "pruned_kind": s.pruned_kind}


# ---------------------------------------------------------------------------
# torch-facing wrappers
# ---------------------------------------------------------------------------

def _torch():
    import torch
    return torch


def _dev_matrix(x, name):
    torch = _torch()
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) torch tensor" % name)
    if x.dtype != torch.float32 or x.dim() != 2 or not x.is_contiguous():
        raise TypeError("%s must be a contiguous 2-D float32 tensor" % name)
    return x


class Workspace:
    """Reusable device workspace (torch uint8 buffer, grown on demand).

    The sequence operators return before their work is done, so that each stream has a buffer of its
    own: calls on one stream follow each other in it, calls on two may run at once.  A graph replays
    into the buffer that it was captured with, so that one that grew stays too, as long as this
    object, which the program keeps as long as the graph.  (Its replays share that buffer: one at a
    time, and not while other calls run on the stream that it was captured on.)"""

    def __init__(self, device=None):
        self.buf = None
        self.device = device
        self._queued = {}  # (device, stream) -> buffers of calls that do not wait, the last in use

    def get(self, nbytes: int, device):
        torch = _torch()
        if self.buf is None or self.buf.numel() < nbytes or self.buf.device != device:
            self.buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        return self.buf

    def get_queued(self, nbytes: int, device):
        """The buffer of the current stream, for a call that does not wait."""
        index = device.index
        bufs = self._queued.get((index, _seq().stream(index)))
        if bufs is None:
            bufs = self._queued.setdefault((index, _seq().stream(index)), [])
        elif bufs[-1].numel() >= nbytes:
            return bufs[-1]
        # At least twice as large as the last: all that are kept are no more than that again.
        least = 2 * bufs[-1].numel() if bufs else 256
        bufs.append(_torch().empty(max(nbytes, least), dtype=_seq().u8, device=device))
        return bufs[-1]


class FixedWorkspace:
    """A device workspace of a fixed size chosen by the caller.  The library
    plans its query blocks to fit it (automatic batching sized to memory);
    a workspace below the fixed buffers plus one 32-row block is an error.
    It is one buffer: sequence operators that use it run on one stream."""

    def __init__(self, nbytes: int, device="cuda:0"):
        torch = _torch()
        self.buf = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)

    def get(self, nbytes: int, device):
        return self.buf


def _ws(workspace, nbytes, device):
    """(buffer, pointer, size) of a workspace of at least nbytes.

    The caller must hold the returned buffer until the library call returns:
    a temporary workspace would otherwise go back to torch's caching
    allocator, which may hand the same memory to the next output tensor.
    """
    if workspace is None:
        workspace = Workspace()
    buf = workspace.get(nbytes, device)
    return buf, ctypes.c_void_p(buf.data_ptr()), ctypes.c_size_t(buf.numel())


def _stream(stream):
    torch = _torch()
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _p(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def tod_knn(xq, xr, k: int, opts=None, workspace=None, stream=None, stats=None):
    """k nearest rows of xr for every row of xq -> (idx int64 [nq,k], dist fp32 [nq,k])."""
    torch = _torch()
    _dev_matrix(xq, "xq")
    _dev_matrix(xr, "xr")
    nq, d = xq.shape
    nr = xr.shape[0]
    if xr.shape[1] != d:
        raise ValueError("xq and xr must have the same number of columns")
    idx = torch.empty((nq, k), dtype=torch.int64, device=xq.device)
    dist = torch.empty((nq, k), dtype=torch.float32, device=xq.device)
    need = tod_workspace_size(nq, nr, d, k, False, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, xq.device)
    st = _lib.tod_knn(_p(xq), nq, _p(xr), nr, d, int(k),
                      ctypes.byref(opts) if opts is not None else None, wsp, wsn,
                      _stream(stream), _p(idx), _p(dist),
                      ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_knn")
    return idx, dist


NOALLOC_SCRATCH_BYTES = 64 << 20  # TOD_NOALLOC_SCRATCH_BYTES of include/tod.h


def tod_knn_noalloc(xq, xr, k: int, opts=None, stream=None, stats=None, out=None):
    """tod_knn with the library's static scratch as its workspace (no device
    allocation inside the call) -> (idx int64 [nq,k], dist fp32 [nq,k]).
    out: optional preallocated (idx, dist) tensors, so that the caller's side
    allocates nothing either."""
    torch = _torch()
    _dev_matrix(xq, "xq")
    _dev_matrix(xr, "xr")
    nq, d = xq.shape
    nr = xr.shape[0]
    if xr.shape[1] != d:
        raise ValueError("xq and xr must have the same number of columns")
    if out is None:
        idx = torch.empty((nq, k), dtype=torch.int64, device=xq.device)
        dist = torch.empty((nq, k), dtype=torch.float32, device=xq.device)
    else:
        idx, dist = out
        if (tuple(idx.shape) != (nq, k) or idx.dtype != torch.int64 or not idx.is_contiguous()
                or tuple(dist.shape) != (nq, k) or dist.dtype != torch.float32
                or not dist.is_contiguous()):
            raise ValueError("out must be contiguous (int64 [nq,k], fp32 [nq,k]) tensors")
    st = _lib.tod_knn_noalloc(_p(xq), nq, _p(xr), nr, d, int(k),
                              ctypes.byref(opts) if opts is not None else None,
                              _stream(stream), _p(idx), _p(dist),
                              ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_knn_noalloc")
    return idx, dist


def tod_knn_score(x, k: int, opts=None, workspace=None, stream=None, stats=None,
                  return_lists: bool = False):
    """kNN-OD score of every row of x (self excluded); optionally the lists too."""
    torch = _torch()
    _dev_matrix(x, "x")
    n, d = x.shape
    score = torch.empty((n,), dtype=torch.float32, device=x.device)
    idx = dist = None
    if return_lists:
        idx = torch.empty((n, k), dtype=torch.int64, device=x.device)
        dist = torch.empty((n, k), dtype=torch.float32, device=x.device)
    need = tod_workspace_size(n, n, d, k, False, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, x.device)
    st = _lib.tod_knn_score(_p(x), n, d, int(k), ctypes.byref(opts) if opts is not None else None,
                            wsp, wsn, _stream(stream), _p(score), _p(idx), _p(dist),
                            ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_knn_score")
    return (score, idx, dist) if return_lists else score


def tod_lof(x, k: int, opts=None, workspace=None, stream=None, stats=None,
            return_lists: bool = False, out=None):
    """LOF and kNN-OD scores of every row of x -> (lof fp32 [n], knn_score fp32 [n][, idx, dist])."""
    torch = _torch()
    _dev_matrix(x, "x")
    n, d = x.shape
    if out is None:
        lof = torch.empty((n,), dtype=torch.float32, device=x.device)
        score = torch.empty((n,), dtype=torch.float32, device=x.device)
    else:
        lof, score = out
    idx = dist = None
    if return_lists:
        idx = torch.empty((n, k), dtype=torch.int64, device=x.device)
        dist = torch.empty((n, k), dtype=torch.float32, device=x.device)
    need = tod_workspace_size(n, n, d, k, True, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, x.device)
    st = _lib.tod_lof(_p(x), n, d, int(k), ctypes.byref(opts) if opts is not None else None,
                      wsp, wsn, _stream(stream), _p(lof), _p(score), _p(idx), _p(dist),
                      ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_lof")
    return (lof, score, idx, dist) if return_lists else (lof, score)


def tod_lof_ties_workspace_size(n: int, d: int, k: int, capacity: int, opts=None) -> int:
    return int(_lib.tod_lof_ties_workspace_size(int(n), int(d), int(k), int(capacity),
                                                ctypes.byref(opts) if opts is not None else None))


def tod_lof_ties(x, k: int, opts=None, capacity=None, grow: bool = True, workspace=None,
                 stream=None, stats=None):
    """LOF on tie-inclusive k-distance neighbourhoods -> (lof fp32 [n], count int32 [n]).

    ``capacity`` is the number of (point, neighbour) pairs the workspace is
    sized for (default n k + n + 2^16); if the neighbourhoods hold more and
    ``grow`` is set, the workspace is resized to the count the library
    reports and the call is made once more, else TodError(TOD_ERR_CAPACITY)
    is raised.
    """
    torch = _torch()
    _dev_matrix(x, "x")
    n, d = x.shape
    lof = torch.empty((n,), dtype=torch.float32, device=x.device)
    count = torch.empty((n,), dtype=torch.int32, device=x.device)
    st = stats if stats is not None else new_stats()
    optp = ctypes.byref(opts) if opts is not None else None
    cap = int(capacity) if capacity is not None else n * int(k) + n + (1 << 16)
    for _ in range(2):
        need = tod_lof_ties_workspace_size(n, d, k, cap, opts)
        if need == 0:  # arguments the size query rejects: let the call report why
            need = 256
        wsbuf, wsp, wsn = _ws(workspace, need, x.device)
        rc = _lib.tod_lof_ties(_p(x), n, d, int(k), cap, optp, wsp, wsn, _stream(stream),
                               _p(lof), _p(count), ctypes.byref(st))
        if rc != TOD_ERR_CAPACITY or not grow:
            break
        cap = int(st.pairs_in_range)
    _check(rc, "tod_lof_ties")
    del wsbuf
    return lof, count


def tod_knn_decision(xq, xr, k: int, opts=None, workspace=None, stream=None, stats=None,
                     return_lists: bool = False):
    """kNN-OD scores of new points xq against the fitted set xr (nothing excluded)."""
    torch = _torch()
    _dev_matrix(xq, "xq")
    _dev_matrix(xr, "xr")
    nq, d = xq.shape
    nr = xr.shape[0]
    if xr.shape[1] != d:
        raise ValueError("xq and xr must have the same number of columns")
    score = torch.empty((nq,), dtype=torch.float32, device=xq.device)
    idx = dist = None
    if return_lists:
        idx = torch.empty((nq, k), dtype=torch.int64, device=xq.device)
        dist = torch.empty((nq, k), dtype=torch.float32, device=xq.device)
    need = tod_workspace_size(nq, nr, d, k, 0, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, xq.device)
    st = _lib.tod_knn_decision(_p(xq), nq, _p(xr), nr, d, int(k),
                               ctypes.byref(opts) if opts is not None else None, wsp, wsn,
                               _stream(stream), _p(score), _p(idx), _p(dist),
                               ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_knn_decision")
    return (score, idx, dist) if return_lists else score


def tod_knn_classify(xq, xr, labels_r, k: int, n_classes: int, opts=None, workspace=None,
                     stream=None, stats=None):
    """Majority-vote class of every row of xq among its k nearest rows of xr -> int32 [nq]."""
    torch = _torch()
    _dev_matrix(xq, "xq")
    _dev_matrix(xr, "xr")
    if (not isinstance(labels_r, torch.Tensor) or not labels_r.is_cuda
            or labels_r.dtype != torch.int32 or labels_r.dim() != 1
            or labels_r.shape[0] != xr.shape[0] or not labels_r.is_contiguous()):
        raise TypeError("labels_r must be a contiguous int32 CUDA tensor of length nr")
    nq, d = xq.shape
    nr = xr.shape[0]
    pred = torch.empty((nq,), dtype=torch.int32, device=xq.device)
    need = tod_workspace_size(nq, nr, d, k, 2, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, xq.device)
    st = _lib.tod_knn_classify(_p(xq), nq, _p(xr), nr, d, int(k), _p(labels_r), int(n_classes),
                               ctypes.byref(opts) if opts is not None else None, wsp, wsn,
                               _stream(stream), _p(pred),
                               ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_knn_classify")
    return pred


def tod_abod(x, k: int, opts=None, workspace=None, stream=None, stats=None,
             return_lists: bool = False):
    """ABOD score (mean neighbour-pair cosine) of every row of x (self excluded)."""
    torch = _torch()
    _dev_matrix(x, "x")
    n, d = x.shape
    score = torch.empty((n,), dtype=torch.float32, device=x.device)
    idx = dist = None
    if return_lists:
        idx = torch.empty((n, k), dtype=torch.int64, device=x.device)
        dist = torch.empty((n, k), dtype=torch.float32, device=x.device)
    need = tod_workspace_size(n, n, d, k, 1, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, x.device)
    st = _lib.tod_abod(_p(x), n, d, int(k), ctypes.byref(opts) if opts is not None else None,
                       wsp, wsn, _stream(stream), _p(score), _p(idx), _p(dist),
                       ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_abod")
    return (score, idx, dist) if return_lists else score


def tod_cof(x, k: int, opts=None, workspace=None, stream=None, stats=None,
            return_lists: bool = False):
    """COF of every row of x (self excluded) -> (cof fp32 [n], knn_score fp32 [n][, idx, dist])."""
    torch = _torch()
    _dev_matrix(x, "x")
    n, d = x.shape
    cof = torch.empty((n,), dtype=torch.float32, device=x.device)
    score = torch.empty((n,), dtype=torch.float32, device=x.device)
    idx = dist = None
    if return_lists:
        idx = torch.empty((n, k), dtype=torch.int64, device=x.device)
        dist = torch.empty((n, k), dtype=torch.float32, device=x.device)
    need = tod_workspace_size(n, n, d, k, 1, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, x.device)
    st = _lib.tod_cof(_p(x), n, d, int(k), ctypes.byref(opts) if opts is not None else None,
                      wsp, wsn, _stream(stream), _p(cof), _p(score), _p(idx), _p(dist),
                      ctypes.byref(stats) if stats is not None else None)
    _check(st, "tod_cof")
    return (cof, score, idx, dist) if return_lists else (cof, score)


def tod_nwr_workspace_size(nq: int, nr: int, d: int, opts=None) -> int:
    return int(_lib.tod_nwr_workspace_size(int(nq), int(nr), int(d),
                                           ctypes.byref(opts) if opts is not None else None))


def tod_nwr(xq, xr, phi: float, opts=None, workspace=None, stream=None, stats=None,
            capacity=None, with_dist: bool = True, count_only: bool = False,
            workspace_bytes=None):
    """Neighbours within range phi -> (row_ptr int64 [nq+1], idx int64 [total], dist fp32 [total]).

    With count_only, only row_ptr is computed (idx and dist are None).  The
    outputs are allocated with ``capacity`` entries (default 64 per query
    row); if the pairs in range do not fit, they are reallocated to the
    total the library reports and the call is made once more.
    ``workspace_bytes`` overrides the workspace size (candidate room).
    """
    torch = _torch()
    _dev_matrix(xq, "xq")
    _dev_matrix(xr, "xr")
    nq, d = xq.shape
    nr = xr.shape[0]
    if xr.shape[1] != d:
        raise ValueError("xq and xr must have the same number of columns")
    need = int(workspace_bytes) if workspace_bytes is not None else \
        tod_nwr_workspace_size(nq, nr, d, opts)
    wsbuf, wsp, wsn = _ws(workspace, need, xq.device)
    row_ptr = torch.empty((nq + 1,), dtype=torch.int64, device=xq.device)
    total = ctypes.c_int64(0)
    optp = ctypes.byref(opts) if opts is not None else None
    stp = ctypes.byref(stats) if stats is not None else None
    if count_only:
        st = _lib.tod_nwr(_p(xq), nq, _p(xr), nr, d, float(phi), optp, wsp, wsn, _stream(stream),
                          _p(row_ptr), 0, None, None, ctypes.byref(total), stp)
        _check(st, "tod_nwr")
        return row_ptr, None, None
    cap = 64 * nq if capacity is None else int(capacity)
    for _ in range(2):
        idx = torch.empty((max(cap, 1),), dtype=torch.int64, device=xq.device)
        dist = torch.empty((max(cap, 1),), dtype=torch.float32, device=xq.device) \
            if with_dist else None
        st = _lib.tod_nwr(_p(xq), nq, _p(xr), nr, d, float(phi), optp, wsp, wsn, _stream(stream),
                          _p(row_ptr), cap, _p(idx), _p(dist), ctypes.byref(total), stp)
        if st != TOD_ERR_CAPACITY:
            break
        cap = int(total.value)
    _check(st, "tod_nwr")
    n = int(total.value)
    return row_ptr, idx[:n], (dist[:n] if dist is not None else None)


def tod_loci_workspace_size(n: int, d: int, n_radii: int, capacity: int, opts=None) -> int:
    return int(_lib.tod_loci_workspace_size(int(n), int(d), int(n_radii), int(capacity),
                                            ctypes.byref(opts) if opts is not None else None))


def tod_loci(x, radii, alpha: float = 0.5, n_min: int = 20, k_sigma: float = 3.0, opts=None,
             capacity=None, grow: bool = True, workspace=None, stream=None, stats=None,
             return_all: bool = False):
    """LOCI at the ladder of sampling radii -> (score fp64 [n], flag int32 [n]).

    With return_all, a third element holds n_alpha, n_r (int32 [n, L]), mdef
    and sigma_mdef (fp64 [n, L]).  ``capacity`` is the number of pairs within
    the largest radius (self pairs included) the workspace is sized for
    (default 64 per row); if more are in range and ``grow`` is set, the
    workspace is resized to the count the library reports and the call is
    made once more, else TodError(TOD_ERR_CAPACITY) is raised.
    """
    torch = _torch()
    _dev_matrix(x, "x")
    n, d = x.shape
    rad = [float(r) for r in radii]
    nl = len(rad)
    rarr = (ctypes.c_double * max(nl, 1))(*rad)
    dev = x.device
    score = torch.empty((n,), dtype=torch.float64, device=dev)
    flag = torch.empty((n,), dtype=torch.int32, device=dev)
    extra = None
    if return_all:
        extra = {"n_alpha": torch.empty((n, nl), dtype=torch.int32, device=dev),
                 "n_r": torch.empty((n, nl), dtype=torch.int32, device=dev),
                 "mdef": torch.empty((n, nl), dtype=torch.float64, device=dev),
                 "sigma_mdef": torch.empty((n, nl), dtype=torch.float64, device=dev)}
    st = stats if stats is not None else new_stats()
    optp = ctypes.byref(opts) if opts is not None else None
    cap = int(capacity) if capacity is not None else 64 * n
    for _ in range(2):
        need = tod_loci_workspace_size(n, d, nl, cap, opts)
        if need == 0:  # arguments the size query rejects: let the call report why
            need = 256
        wsbuf, wsp, wsn = _ws(workspace, need, dev)
        rc = _lib.tod_loci(_p(x), n, d, rarr, nl, float(alpha), int(n_min), float(k_sigma), cap,
                           optp, wsp, wsn, _stream(stream), _p(score), _p(flag),
                           _p(extra["n_alpha"]) if extra else None,
                           _p(extra["n_r"]) if extra else None,
                           _p(extra["mdef"]) if extra else None,
                           _p(extra["sigma_mdef"]) if extra else None, ctypes.byref(st))
        if rc != TOD_ERR_CAPACITY or not grow:
            break
        cap = int(st.pairs_in_range)
    _check(rc, "tod_loci")
    del wsbuf
    return (score, flag, extra) if return_all else (score, flag)


# ---------------------------------------------------------------------------
# sequence operators: queued on the stream, not waited for; forward only
# ---------------------------------------------------------------------------

class _Seq:
    """What the calls below need of torch, looked up once: they queue microseconds of work, and
    the program's time between two calls counts as much as the GPU's."""

    def __init__(self):
        torch = _torch()
        self.f32, self.i32, self.i64 = (torch.float32,), (torch.int32,), (torch.int64,)
        self.u8 = torch.uint8
        self.half = (torch.float16, torch.bfloat16)
        self.fp16 = torch.float16
        self.stream = torch._C._cuda_getCurrentRawStream  # (device index) -> hipStream_t
        self.device = torch._C._cuda_getDevice
        self.guard = torch.cuda.device
        self.on = torch.cuda.stream
        self.current = torch.cuda.current_stream
        self.gradients = torch.is_grad_enabled


_seq_env = None


def _seq():
    global _seq_env
    if _seq_env is None:
        _seq_env = _Seq()
    return _seq_env


def _index_of(x, name):
    """Device index of a call's first tensor."""
    if not isinstance(x, _torch().Tensor) or not x.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) torch tensor" % name)
    return x.get_device()


def _want(x, name, dtypes, dim, index, contiguous=True):
    try:
        if (x.get_device() == index and x.dtype in dtypes and x.dim() == dim
                and (not contiguous or x.is_contiguous())):
            if x.requires_grad and _seq().gradients():
                raise ValueError("%s requires a gradient, which this operator does not pass on: "
                                 "detach it or call under torch.no_grad()" % name)
            return
    except AttributeError:
        pass
    if _index_of(x, name) != index:
        raise ValueError("%s must be on the other tensors' device" % name)
    raise TypeError("%s must be a %s%d-dimensional tensor of dtype %s" % (
        name, "contiguous " if contiguous else "", dim, " or ".join(str(d) for d in dtypes)))


def _strides(x, name):
    """(token stride, head stride) of a [tokens, heads, dim] tensor for the library."""
    tokens, heads, dim = x.shape
    row, head, one = x.stride()
    if one != 1 and dim > 1:
        raise TypeError("the elements of a head of %s must be contiguous" % name)
    if (row == 0 and tokens > 1) or (head == 0 and heads > 1):
        raise ValueError("%s is broadcast over tokens or heads" % name)
    return (row if tokens > 1 else 0), (head if heads > 1 else dim)


def _new(like, shape, dtype, stream):
    """An uninitialised tensor that the stream may write at once.

    torch's allocator hands memory that was freed on a stream to that stream's next tensor, while
    its work may still use it: the memory has to come from the stream that the call runs on.  The
    caller reads it on the current one."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    env = _seq()
    with env.on(stream):
        out = like.new_empty(shape, dtype=dtype)
    out.record_stream(env.current(like.device))
    return out


def _queue(where, fn, index, stream, tensors, *args):
    """fn(*args, stream pointer, ...) on the stream; args holds _STREAM in the stream's place.

    The work outlives the call, and torch's allocator gives freed memory to the stream that it
    was allocated on: with a stream of the caller's, every tensor is recorded as used there."""
    env = _seq()
    current = env.stream(index)
    at = current
    if stream is not None:
        if stream.device.index != index:
            raise ValueError("the stream belongs to another device than the tensors")
        at = stream.cuda_stream
    args = [at if a is _STREAM else a for a in args]
    if env.device() == index:
        status = fn(*args)
    else:
        with env.guard(index):
            status = fn(*args)
    if status != TOD_OK:
        _check(status, where)
    if at != current:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


_STREAM = object()


def tod_page_map(cached, fresh, free_pages, table, page_rows: int, tokens: int, stream=None):
    """Pages and slots of every sequence's new tokens.

    cached, fresh: int32 [n_seq]; free_pages: int32 [n_free]; table: int32 [n_seq, cols],
    updated in place; tokens: the number of new tokens (a larger number pads the outputs; with 0 the
    table stays as it is).
    -> (row_start int32 [n_seq + 1], slot int64 [tokens], pos int32 [tokens],
        used int64 [2]: pages needed, which free_pages gives as far as it goes, and new tokens left
        without a slot)
    """
    dev = _index_of(cached, "cached")
    env = _seq()
    _want(cached, "cached", env.i32, 1, dev)
    _want(fresh, "fresh", env.i32, 1, dev)
    _want(free_pages, "free_pages", env.i32, 1, dev)
    _want(table, "table", env.i32, 2, dev)
    n, cols = table.shape
    if fresh.shape[0] != n or cached.shape[0] != n:
        raise ValueError("cached, fresh and table must have one row per sequence")
    tokens = int(tokens)
    if tokens == 0:
        with env.on(stream):
            used = fresh.new_zeros((2,), dtype=env.i64[0])
            used[1] = fresh.clamp(min=0).sum()  # all of them are left out
            row_start = fresh.new_zeros((n + 1,))
        if stream is not None:  # (see _queue and _new)
            fresh.record_stream(stream)
            for t in (row_start, used):
                t.record_stream(env.current(dev))
        return row_start, used.new_empty((0,)), fresh.new_empty((0,)), used
    room = max(tokens, 0)
    # One allocation: used, slot (int64), then row_start and pos (int32).
    words = 2 * (2 + room)
    buf = _new(cached, (words + n + 1 + room,), env.i32[0], stream)
    longs = buf[:words].view(env.i64[0])
    used, slot = longs[:2], longs[2:]
    row_start, pos = buf[words:words + n + 1], buf[words + n + 1:]
    base = buf.data_ptr()
    rows = base + 4 * words
    _queue("tod_page_map", _lib.tod_page_map, dev, stream,
           (cached, fresh, free_pages, table, buf),
           cached.data_ptr(), fresh.data_ptr(), n, free_pages.data_ptr(), free_pages.shape[0],
           int(page_rows), table.data_ptr(), cols, tokens, _STREAM, rows, base + 16,
           rows + 4 * (n + 1), base)
    return row_start, slot, pos, used


def _pages(k_pages, v_pages, dtypes, index):
    _want(k_pages, "k_pages", dtypes, 4, index)
    _want(v_pages, "v_pages", (k_pages.dtype,), 4, index)
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    return k_pages.shape


def tod_page_write(k, v, slot, k_pages, v_pages, stream=None):
    """Write k, v [tokens, kv_heads, dim] into their slots (int64 [tokens], negative: none) of
    k_pages, v_pages [n_pages, kv_heads, page_rows, dim], in place."""
    dev = _index_of(k, "k")
    env = _seq()
    _want(k, "k", env.half, 3, dev, False)
    _want(v, "v", (k.dtype,), 3, dev, False)
    _want(slot, "slot", env.i64, 1, dev)
    n_pages, kv_heads, page_rows, dim = _pages(k_pages, v_pages, (k.dtype,), dev)
    tokens = slot.shape[0]
    if k.shape != (tokens, kv_heads, dim) or v.shape != k.shape:
        raise ValueError("k and v must be [%d, %d, %d] as slot and the pages are"
                         % (tokens, kv_heads, dim))
    if tokens == 0:
        return
    (kr, kh), (vr, vh) = _strides(k, "k"), _strides(v, "v")
    _queue("tod_page_write", _lib.tod_page_write, dev, stream, (k, v, slot, k_pages, v_pages),
           k.data_ptr(), v.data_ptr(), tokens, kv_heads, dim, kr, kh, vr, vh, slot.data_ptr(),
           k_pages.data_ptr(), v_pages.data_ptr(), n_pages, page_rows, _STREAM)


def _attn(q, kv_heads, causal, scale, k=None, v=None):
    _, heads, dim = q.shape
    if scale is None:
        scale = 0.0  # the library's default
    else:
        scale = ctypes.c_float(scale).value
        if not scale > 0.0:
            raise ValueError("scale must be positive, and in 32 bits too")
    kr = kh = vr = vh = 0
    if k is not None:
        (kr, kh), (vr, vh) = _strides(k, "k"), _strides(v, "v")
    qr, qh = _strides(q, "q")
    return tod_attn(_ATTN_SIZE, PREC_FP16 if q.dtype == _seq().fp16 else PREC_BF16, heads,
                    kv_heads, dim, 1 if causal else 0, scale, qr, qh, kr, kh, vr, vh)


_ATTN_SIZE = ctypes.sizeof(tod_attn)


def _attn_outputs(q, out, return_lse, stream):
    if out is None:
        out = _new(q, q.shape, q.dtype, stream)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != q.device \
            or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of q's shape, dtype and device")
    else:
        _want(out, "out", (q.dtype,), 3, q.get_device())
    return out, (_new(q, q.shape[:2], _seq().f32[0], stream) if return_lse else None)


def _attn_ws(workspace, nbytes, like, stream):
    """A workspace of nbytes at least that the stream may write at once (see _new)."""
    if workspace is None:
        return _new(like, (max(nbytes, 256),), _seq().u8, stream)
    get = workspace.get_queued if isinstance(workspace, Workspace) else workspace.get
    if stream is None:
        return get(nbytes, like.device)
    with _seq().on(stream):
        return get(nbytes, like.device)


@functools.lru_cache(maxsize=1024)
def _attn_room(heads, kv_heads, dim, tokens, n_seq, max_fresh):
    a = tod_attn()
    _lib.tod_default_attn(ctypes.byref(a), heads, kv_heads, dim, PREC_FP16)
    return int(_lib.tod_attn_workspace_size(ctypes.byref(a), tokens, n_seq, max_fresh))


def tod_attn_workspace_size(heads: int, kv_heads: int, dim: int, tokens: int, n_seq: int,
                            max_fresh=None) -> int:
    """Workspace bytes of tod_attn_prompt and tod_attn_paged (0: sizes that they refuse)."""
    return _attn_room(int(heads), int(kv_heads), int(dim), int(tokens), int(n_seq),
                      int(tokens if max_fresh is None else max_fresh))


def tod_attn_prompt(q, k, v, row_start, causal: bool = True, scale=None, workspace=None,
                    stream=None, out=None, return_lse: bool = False):
    """Attention over whole packed prompts.

    q [tokens, heads, dim], k, v [tokens, kv_heads, dim] (fp16 or bf16, any token and head
    strides that are multiples of 8); row_start int32 [n_seq + 1].
    -> out [tokens, heads, dim], and with return_lse the softmax's log sums fp32 [tokens, heads].
    """
    dev = _index_of(q, "q")
    env = _seq()
    _want(q, "q", env.half, 3, dev, False)
    _want(k, "k", (q.dtype,), 3, dev, False)
    _want(v, "v", (q.dtype,), 3, dev, False)
    _want(row_start, "row_start", env.i32, 1, dev)
    tokens, heads, dim = q.shape
    kv_heads, n = k.shape[1], row_start.shape[0] - 1
    if k.shape != (tokens, kv_heads, dim) or v.shape != k.shape:
        raise ValueError("k and v must be [tokens, kv_heads, dim] with q's tokens and dim")
    a = _attn(q, kv_heads, causal, scale, k, v)
    out, lse = _attn_outputs(q, out, return_lse, stream)
    if tokens == 0:
        return (out, lse) if return_lse else out
    buf = _attn_ws(workspace, _attn_room(heads, kv_heads, dim, tokens, n, tokens), q, stream)
    _queue("tod_attn_prompt", _lib.tod_attn_prompt, dev, stream,
           (q, k, v, row_start, out, lse, buf),
           ctypes.byref(a), q.data_ptr(), k.data_ptr(), v.data_ptr(), tokens,
           row_start.data_ptr(), n, buf.data_ptr(), buf.numel(), _STREAM, out.data_ptr(),
           lse.data_ptr() if return_lse else None)
    return (out, lse) if return_lse else out


def tod_attn_paged(q, k_pages, v_pages, table, row_start, cached, max_fresh=None, scale=None,
                   workspace=None, stream=None, out=None, return_lse: bool = False):
    """Attention of every sequence's new tokens over its pages.

    q [tokens, heads, dim]; k_pages, v_pages [n_pages, kv_heads, page_rows, dim], the new tokens'
    keys and values written; table int32 [n_seq, cols]; row_start int32 [n_seq + 1]; cached int32
    [n_seq]: tokens in the cache before this step.  max_fresh: the most new tokens of a sequence,
    where the caller knows it.
    -> out [tokens, heads, dim], and with return_lse the softmax's log sums fp32 [tokens, heads].
    """
    dev = _index_of(q, "q")
    env = _seq()
    _want(q, "q", env.half, 3, dev, False)
    n_pages, kv_heads, page_rows, dim = _pages(k_pages, v_pages, (q.dtype,), dev)
    _want(table, "table", env.i32, 2, dev)
    _want(row_start, "row_start", env.i32, 1, dev)
    _want(cached, "cached", env.i32, 1, dev)
    tokens, heads, _ = q.shape
    n, cols = table.shape
    if q.shape[2] != dim:
        raise ValueError("q and the pages must have the same dim")
    if cached.shape[0] != n or row_start.shape[0] != n + 1:
        raise ValueError("table, row_start and cached must describe the same sequences")
    a = _attn(q, kv_heads, True, scale)
    out, lse = _attn_outputs(q, out, return_lse, stream)
    if tokens == 0:
        return (out, lse) if return_lse else out
    fresh = tokens if max_fresh is None else int(max_fresh)
    buf = _attn_ws(workspace, _attn_room(heads, kv_heads, dim, tokens, n, fresh), q, stream)
    _queue("tod_attn_paged", _lib.tod_attn_paged, dev, stream,
           (q, k_pages, v_pages, table, row_start, cached, out, lse, buf),
           ctypes.byref(a), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), n_pages,
           page_rows, table.data_ptr(), cols, row_start.data_ptr(), cached.data_ptr(), n, tokens,
           fresh, buf.data_ptr(), buf.numel(), _STREAM, out.data_ptr(),
           lse.data_ptr() if return_lse else None)
    return (out, lse) if return_lse else out


class Cache4:
    """A paged key / value cache of 4-bit rows, from its tensors (contiguous, uint8):

    k_codes, v_codes [n_pages, kv_heads, page_rows, dim / 2]: two codes a byte, the even element's
    in the low half; k_scales, v_scales [n_pages, kv_heads, page_rows, dim / 32]: the scale of a
    block of 32 elements, 2^(byte - 127).  Cache4.zeros makes them.  dim is a multiple of 32.
    """

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        self._index = _index_of(k_codes, "k_codes")
        u8 = (_seq().u8,)
        for x, name in ((k_codes, "k_codes"), (k_scales, "k_scales"), (v_codes, "v_codes"),
                        (v_scales, "v_scales")):
            _want(x, name, u8, 4, self._index)
        n, heads, rows, half = k_codes.shape
        if half % 16:
            raise ValueError("dim must be a multiple of 32")
        if v_codes.shape != k_codes.shape or k_scales.shape != (n, heads, rows, half // 16) \
                or v_scales.shape != k_scales.shape:
            raise ValueError("codes must be [pages, heads, rows, dim / 2] and scales "
                             "[pages, heads, rows, dim / 32], the same for keys and values")
        self._tensors = (k_codes, k_scales, v_codes, v_scales)
        self.n_pages, self.kv_heads, self.page_rows, self.dim = n, heads, rows, 2 * half

    @classmethod
    def zeros(cls, n_pages: int, kv_heads: int, page_rows: int, dim: int, device="cuda:0"):
        torch = _torch()
        if dim % 32:
            raise ValueError("dim must be a multiple of 32")
        return cls(*(torch.zeros((n_pages, kv_heads, page_rows, dim // per), dtype=torch.uint8,
                                 device=device) for per in (2, 32, 2, 32)))

    k_codes = property(lambda self: self._tensors[0])
    k_scales = property(lambda self: self._tensors[1])
    v_codes = property(lambda self: self._tensors[2])
    v_scales = property(lambda self: self._tensors[3])

    def _arg(self, index):
        if self._index != index:
            raise ValueError("the cache must be on the other tensors' device")
        kc, ks, vc, vs = self._tensors
        return tod_cache4(_CACHE4_SIZE, self.page_rows, self.n_pages, kc.data_ptr(), vc.data_ptr(),
                          ks.data_ptr(), vs.data_ptr())


_CACHE4_SIZE = ctypes.sizeof(tod_cache4)
_APPEND_SIZE = ctypes.sizeof(tod_append)


def _append(q, k, v, pos, slot, rates, kv_heads, dim, interleaved, stream, out):
    """Checks that both appends share -> (device index, q_out, tod_append)."""
    dev = _index_of(q, "q")
    env = _seq()
    _want(q, "q", env.half, 3, dev, False)
    _want(k, "k", (q.dtype,), 3, dev, False)
    _want(v, "v", (q.dtype,), 3, dev, False)
    _want(pos, "pos", env.i32, 1, dev)
    _want(slot, "slot", env.i64, 1, dev)
    _want(rates, "rates", env.f32, 1, dev)
    tokens, heads, _ = q.shape
    if q.shape[2] != dim or k.shape != (tokens, kv_heads, dim) or v.shape != k.shape:
        raise ValueError("q must be [tokens, heads, %d] and k and v [tokens, %d, %d] as the cache is"
                         % (dim, kv_heads, dim))
    if pos.shape[0] != tokens or slot.shape[0] != tokens:
        raise ValueError("pos and slot must have one entry per token")
    rotary = 2 * rates.shape[0]
    if rotary > dim:
        raise ValueError("rates must have at most dim / 2 entries")
    (qr, qh), (kr, kh), (vr, vh) = _strides(q, "q"), _strides(k, "k"), _strides(v, "v")
    out, _ = _attn_outputs(q, out, False, stream)
    return dev, out, tod_append(_APPEND_SIZE, PREC_FP16 if q.dtype == env.fp16 else PREC_BF16,
                                heads, kv_heads, dim, rotary, 1 if interleaved else 0, qr, qh, kr,
                                kh, vr, vh)


def tod_page_append(q, k, v, pos, slot, rates, k_pages, v_pages, interleaved: bool = False,
                    stream=None, out=None):
    """Rotate q and k by position, and write k and v into their slots of 16-bit pages.

    q [tokens, heads, dim], k, v [tokens, kv_heads, dim] (fp16 or bf16, strides as of
    tod_attn_prompt); pos int32 and slot int64 [tokens], as of tod_page_map; rates fp32 [r / 2]:
    the angle of a step of one position, for the pairs (i, i + r / 2) of a head's first r elements,
    or (2 i, 2 i + 1) with interleaved; k_pages, v_pages as in tod_page_write, written in place.
    -> the rotated q [tokens, heads, dim]
    """
    _, kv_heads, page_rows, dim = _pages(k_pages, v_pages, _seq().half, _index_of(q, "q"))
    dev, out, a = _append(q, k, v, pos, slot, rates, kv_heads, dim, interleaved, stream, out)
    if k_pages.dtype != q.dtype:
        raise TypeError("k_pages must have q's dtype")
    tokens = q.shape[0]
    if tokens == 0:
        return out
    _queue("tod_page_append", _lib.tod_page_append, dev, stream,
           (q, k, v, pos, slot, rates, k_pages, v_pages, out),
           ctypes.byref(a), q.data_ptr(), k.data_ptr(), v.data_ptr(), tokens, pos.data_ptr(),
           rates.data_ptr(), slot.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
           k_pages.shape[0], page_rows, _STREAM, out.data_ptr())
    return out


def tod_page_append4(q, k, v, pos, slot, rates, cache, interleaved: bool = False, stream=None,
                     out=None):
    """Rotate q and k by position, and write k and v into their slots of a 4-bit cache (Cache4).

    Arguments as in tod_page_append.  A block of 32 elements with the largest magnitude a gets the
    smallest scale 2^e with a <= 7 2^e, and its elements the nearest of the codes' values.
    -> the rotated q [tokens, heads, dim]
    """
    dev, out, a = _append(q, k, v, pos, slot, rates, cache.kv_heads, cache.dim, interleaved, stream,
                          out)
    c = cache._arg(dev)
    tokens = q.shape[0]
    if tokens == 0:
        return out
    _queue("tod_page_append4", _lib.tod_page_append4, dev, stream,
           (q, k, v, pos, slot, rates, out) + cache._tensors,
           ctypes.byref(a), q.data_ptr(), k.data_ptr(), v.data_ptr(), tokens, pos.data_ptr(),
           rates.data_ptr(), slot.data_ptr(), ctypes.byref(c), _STREAM, out.data_ptr())
    return out


def tod_page_read4(cache, slot, dtype, stream=None):
    """Rows of a 4-bit cache at the slots (int64 [tokens], negative: zeros), as fp16 or bf16.

    -> k, v [tokens, kv_heads, dim]
    """
    dev = _index_of(slot, "slot")
    env = _seq()
    _want(slot, "slot", env.i64, 1, dev)
    if dtype not in env.half:
        raise TypeError("dtype must be %s" % " or ".join(str(d) for d in env.half))
    c = cache._arg(dev)
    tokens = slot.shape[0]
    out = _new(slot, (2, tokens, cache.kv_heads, cache.dim), dtype, stream)
    k, v = out[0], out[1]
    if tokens == 0:
        return k, v
    _queue("tod_page_read4", _lib.tod_page_read4, dev, stream, (slot, out) + cache._tensors,
           ctypes.byref(c), cache.kv_heads, cache.dim,
           PREC_FP16 if dtype == env.fp16 else PREC_BF16, slot.data_ptr(), tokens, _STREAM,
           k.data_ptr(), v.data_ptr())
    return k, v


@functools.lru_cache(maxsize=1024)
def _attn4_room(heads, kv_heads, dim, tokens, n_seq, max_fresh):
    a = tod_attn()
    _lib.tod_default_attn(ctypes.byref(a), heads, kv_heads, dim, PREC_FP16)
    return int(_lib.tod_attn_paged4_workspace_size(ctypes.byref(a), tokens, n_seq, max_fresh))


def tod_attn_paged4_workspace_size(heads: int, kv_heads: int, dim: int, tokens: int, n_seq: int,
                                   max_fresh=None) -> int:
    """Workspace bytes of tod_attn_paged4 (0: sizes that it refuses)."""
    return _attn4_room(int(heads), int(kv_heads), int(dim), int(tokens), int(n_seq),
                       int(tokens if max_fresh is None else max_fresh))


def tod_attn_paged4(q, cache, table, row_start, cached, max_fresh=None, scale=None, workspace=None,
                    stream=None, out=None, return_lse: bool = False):
    """Attention of every sequence's new tokens over its pages of a 4-bit cache (Cache4).

    Arguments and results as in tod_attn_paged, over the values that the cache's codes stand for.
    """
    dev = _index_of(q, "q")
    env = _seq()
    _want(q, "q", env.half, 3, dev, False)
    _want(table, "table", env.i32, 2, dev)
    _want(row_start, "row_start", env.i32, 1, dev)
    _want(cached, "cached", env.i32, 1, dev)
    tokens, heads, dim = q.shape
    n, cols = table.shape
    kv_heads = cache.kv_heads
    if dim != cache.dim:
        raise ValueError("q and the cache must have the same dim")
    if cached.shape[0] != n or row_start.shape[0] != n + 1:
        raise ValueError("table, row_start and cached must describe the same sequences")
    c = cache._arg(dev)
    a = _attn(q, kv_heads, True, scale)
    out, lse = _attn_outputs(q, out, return_lse, stream)
    if tokens == 0:
        return (out, lse) if return_lse else out
    fresh = tokens if max_fresh is None else int(max_fresh)
    buf = _attn_ws(workspace, _attn4_room(heads, kv_heads, dim, tokens, n, fresh), q, stream)
    _queue("tod_attn_paged4", _lib.tod_attn_paged4, dev, stream,
           (q, table, row_start, cached, out, lse, buf) + cache._tensors,
           ctypes.byref(a), q.data_ptr(), ctypes.byref(c), table.data_ptr(), cols,
           row_start.data_ptr(), cached.data_ptr(), n, tokens, fresh, buf.data_ptr(), buf.numel(),
           _STREAM, out.data_ptr(), lse.data_ptr() if return_lse else None)
    return (out, lse) if return_lse else out


def raw_library():
    """The loaded ctypes library (for ABI tests)."""
    return _lib
