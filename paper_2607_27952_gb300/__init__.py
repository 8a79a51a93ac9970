"""Python binding of liblast (GB300 / sm_103a) -- argument marshalling only.

Every step of the path runs in the CUDA kernels of liblast.so; this module
only turns torch tensors (and, for last_prune_host, host buffers) into pointers
and host offset arrays into the C problem struct.  The handles of the key-value
cache (Rope, Cache, Sequences, PagePool) are such structs too, checked once and
reused by every call on them.  There is no CPU fallback: if
the library is missing, every call raises.

Functions carry the names of the C entry points in include/last.h:
  last_workspace_size, last_scores, last_select, last_select_topk, last_gather,
  last_prune, last_host_workspace_size, last_prune_host, last_scores_rows,
  last_scores_rows_workspace_size, last_scores_noalloc, last_check_bounded_wait,
  last_poll, last_budget, last_status_string, last_error_message,
  last_rope, last_rope_backward, last_cache_workspace_size, last_cache_append,
  last_cache_attention, last_chunk_workspace_size, last_cache_chunk_attention,
  last_cache_diff_attention, last_cache_copy, last_cache_compact, last_pages_init,
  last_pages_take, last_pages_share, last_pages_release.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblast.so")

LAST_OK = 0
LAST_ERR_INVALID_ARG = 1
LAST_ERR_UNSUPPORTED = 2
LAST_ERR_WORKSPACE_TOO_SMALL = 3
LAST_ERR_CUDA = 4
LAST_ERR_DEVICE_INDEX = 5
LAST_ERR_TIMEOUT = 6
LAST_ERR_NO_PAGES = 7

LAST_DTYPE_F32 = 0
LAST_DTYPE_BF16 = 1

LAST_ROPE_HALF = 0
LAST_ROPE_ADJACENT = 1

EXPORTED = ("last_workspace_size", "last_scores", "last_select", "last_gather", "last_prune",
            "last_poll", "last_budget", "last_status_string", "last_error_message",
            "last_scores_noalloc", "last_select_topk", "last_scores_rows",
            "last_scores_rows_workspace_size", "last_check_bounded_wait",
            "last_host_workspace_size", "last_prune_host", "last_rope", "last_rope_backward",
            "last_cache_workspace_size", "last_cache_append", "last_cache_attention",
            "last_cache_copy", "last_cache_compact", "last_pages_init", "last_pages_take",
            "last_pages_share", "last_pages_release", "last_chunk_workspace_size",
            "last_cache_chunk_attention", "last_cache_diff_attention")


class LastError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_status_name(status)}: {message}")
        self.status = status


class _Problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_layers", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("feat_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("cu_seqlens", ctypes.POINTER(ctypes.c_int32)),
                ("vis_start", ctypes.POINTER(ctypes.c_int32)),
                ("cu_vis", ctypes.POINTER(ctypes.c_int32)),
                ("cu_keep", ctypes.POINTER(ctypes.c_int32))]


class _Rotary(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("num_axes", ctypes.c_int32), ("pairs", ctypes.c_int32),
                ("inv_freq", ctypes.POINTER(ctypes.c_float)),
                ("axis", ctypes.POINTER(ctypes.c_int32))]


class _Heads(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("heads", ctypes.c_int32),
                ("in_token", ctypes.c_int64), ("in_head", ctypes.c_int64),
                ("out_token", ctypes.c_int64), ("out_head", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_layers", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


class _Sequences(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("table_stride", ctypes.c_int64), ("page_table", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("key_begin", ctypes.c_void_p)]


class _Difference(ctypes.Structure):
    _fields_ = [("lambda_", ctypes.c_void_p), ("norm_weight", ctypes.c_void_p), ("norm_eps", ctypes.c_float),
                ("out_scale", ctypes.c_float)]


class _PagePool(ctypes.Structure):
    _fields_ = [("num_pages", ctypes.c_int32), ("num_free", ctypes.c_int32),
                ("holders", ctypes.POINTER(ctypes.c_int32)),
                ("free_pages", ctypes.POINTER(ctypes.c_int32))]


_lib = None
_fast = None   # the calls of the cache without ctypes (csrc/marshal.c), where that module has been built


def _load_fast(lib):
    """The marshalling module bound to the library, or None."""
    try:
        import torch
        from . import _marshal
        names = ("last_rope", "last_rope_backward", "last_cache_append", "last_cache_attention", "last_cache_copy",
                 "last_cache_compact", "last_cache_chunk_attention", "last_cache_diff_attention")
        _marshal.bind(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names), torch.float32, torch.bfloat16,
                      torch.int32, torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice)
    except (ImportError, AttributeError, TypeError):   # not built, a torch without these, or built from older sources
        return None
    return _marshal


def load_library(path: str = LIB_PATH):
    """Loads liblast.so (raises if it has not been built)."""
    global _lib, _fast
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'`")
    try:  # share the CUDA runtime that torch loads
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(path)
    P = ctypes.c_void_p
    PP = ctypes.POINTER(_Problem)
    lib.last_workspace_size.argtypes = [PP, ctypes.POINTER(ctypes.c_size_t)]
    lib.last_scores.argtypes = [PP, P, P, P, P, ctypes.c_size_t, P]
    lib.last_select.argtypes = [PP, P, P, P, P, P, ctypes.c_size_t, P]
    lib.last_gather.argtypes = [PP, P, P, P, P, ctypes.c_size_t, P]
    lib.last_select_topk.argtypes = [PP, P, P, P, P, P, ctypes.c_size_t, P]
    PI = ctypes.POINTER(ctypes.c_int32)
    lib.last_scores_rows.argtypes = [PP, PI, PI, P, P, P, P, ctypes.c_size_t, P]
    lib.last_scores_rows_workspace_size.argtypes = [PP, PI, PI, ctypes.POINTER(ctypes.c_size_t)]
    lib.last_prune.argtypes = [PP, P, P, P, P, P, P, P, ctypes.c_size_t, P]
    lib.last_host_workspace_size.argtypes = [PP, ctypes.POINTER(ctypes.c_size_t)]
    lib.last_prune_host.argtypes = [PP, P, P, P, P, P, P, P, ctypes.c_size_t, P]
    lib.last_poll.argtypes = [P, P]
    lib.last_check_bounded_wait.argtypes = [P, P]
    lib.last_scores_noalloc.argtypes = [PP, P, P, P, P]
    lib.last_budget.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
    lib.last_budget.restype = ctypes.c_int32
    lib.last_status_string.argtypes = [ctypes.c_int]
    lib.last_status_string.restype = ctypes.c_char_p
    lib.last_error_message.argtypes = []
    lib.last_error_message.restype = ctypes.c_char_p
    I, L, F, Z = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    PR, PH, PC = (ctypes.POINTER(t) for t in (_Rotary, _Heads, _Cache))
    PS, PG = ctypes.POINTER(_Sequences), ctypes.POINTER(_PagePool)
    lib.last_rope.argtypes = lib.last_rope_backward.argtypes = [PR, I, I, I, P, L, PH, PH, P]
    lib.last_cache_workspace_size.argtypes = [PC, I, I, ctypes.POINTER(Z)]
    lib.last_cache_append.argtypes = [PC, I, PS, I, P, PR, P, L, PH, PH, PH, P, Z, P]
    lib.last_cache_attention.argtypes = [PC, I, PS, I, F, P, L, P, L, P, P, Z, P]
    PD = ctypes.POINTER(_Difference)
    lib.last_chunk_workspace_size.argtypes = [PC, I, ctypes.POINTER(Z)]
    lib.last_cache_chunk_attention.argtypes = [PC, I, PS, I, P, I, F, I, I, P, L, P, L, P, P, Z, P]
    lib.last_cache_diff_attention.argtypes = [PC, I, PS, I, P, I, F, I, I, PD, P, L, P, L, P, Z, P]
    lib.last_cache_copy.argtypes = [PC, I, P, P, P, Z, P]
    lib.last_cache_compact.argtypes = [PC, PS, P, I, L, P, P, P, P, I, P, P, Z, P]
    lib.last_pages_init.argtypes = [PG]
    for name in ("last_pages_take", "last_pages_share", "last_pages_release"):
        getattr(lib, name).argtypes = [PG, I, PI]
    for name in ("last_rope", "last_rope_backward", "last_cache_workspace_size", "last_cache_append",
                 "last_cache_attention", "last_cache_copy", "last_cache_compact",
                 "last_pages_init", "last_pages_take", "last_pages_share", "last_pages_release",
                 "last_chunk_workspace_size", "last_cache_chunk_attention", "last_cache_diff_attention",
                 "last_host_workspace_size", "last_prune_host"):
        getattr(lib, name).restype = ctypes.c_int
    for name in ("last_workspace_size", "last_scores", "last_select", "last_gather",
                 "last_prune", "last_poll", "last_scores_noalloc", "last_select_topk",
                 "last_scores_rows", "last_scores_rows_workspace_size",
                 "last_check_bounded_wait"):
        getattr(lib, name).restype = ctypes.c_int
    _fast = _load_fast(lib)
    _lib = lib
    return lib


def _status_name(st: int) -> str:
    try:
        return load_library().last_status_string(st).decode()
    except ImportError:
        return f"status {st}"


def _check(st: int):
    if st != LAST_OK:
        msg = load_library().last_error_message().decode()
        raise LastError(st, msg)


class Problem:
    """Problem description (include/last.h `last_problem`); keeps its host arrays alive."""

    def __init__(self, *, batch: int, num_layers: int, num_q_heads: int, num_kv_heads: int,
                 head_dim: int, feat_dim: int, dtype: str, cu_seqlens: Optional[Sequence[int]],
                 vis_start: Optional[Sequence[int]], cu_vis: Sequence[int],
                 cu_keep: Sequence[int], softmax_scale: float = 0.0):
        def arr(a):
            return None if a is None else np.ascontiguousarray(np.asarray(a, dtype=np.int32))
        self.arrays = dict(cu_seqlens=arr(cu_seqlens), vis_start=arr(vis_start),
                           cu_vis=arr(cu_vis), cu_keep=arr(cu_keep))
        self.dtype = dtype
        code = {"f32": LAST_DTYPE_F32, "bf16": LAST_DTYPE_BF16}[dtype]

        def ptr(a):
            return None if a is None else a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        self.c = _Problem(batch, num_layers, num_q_heads, num_kv_heads, head_dim, feat_dim, code,
                          float(softmax_scale), ptr(self.arrays["cu_seqlens"]),
                          ptr(self.arrays["vis_start"]), ptr(self.arrays["cu_vis"]),
                          ptr(self.arrays["cu_keep"]))
        self.batch = batch
        self.feat_dim = feat_dim
        self.total_vis = int(self.arrays["cu_vis"][-1])
        self.total_keep = int(self.arrays["cu_keep"][-1])

    @property
    def ref(self):
        return ctypes.byref(self.c)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("liblast takes device tensors")
    if not t.is_contiguous():
        raise ValueError("liblast takes contiguous tensors")
    return t.data_ptr()


def _host_ptr(t) -> Optional[int]:
    """Address of a contiguous host buffer: a CPU torch tensor (pinned for
    asynchronous copies) or a numpy array."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        if not t.flags["C_CONTIGUOUS"]:
            raise ValueError("host buffers must be contiguous")
        return t.ctypes.data
    if t.is_cuda:
        raise ValueError("last_prune_host takes host buffers")
    if not t.is_contiguous():
        raise ValueError("host buffers must be contiguous")
    return t.data_ptr()


def _current_stream() -> int:
    """The current stream's handle without building a torch.cuda.Stream (3 us on a GB300's host)."""
    global _current_stream
    import torch
    get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    torch.cuda.current_stream()      # CUDA is up
    if get is None or device is None:
        _current_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    else:
        _current_stream = lambda: get(device())  # noqa: E731
    return _current_stream()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _ws(ws):
    if isinstance(ws, tuple):
        return ws
    return _ptr(ws), ws.nbytes


def last_workspace_size(problem: Problem) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().last_workspace_size(problem.ref, ctypes.byref(n)))
    return n.value


def _keep_all(problem: Problem) -> Problem:
    """The same problem with every token kept: its workspace size holds no Gram matrices and is
    enough for `problem` whatever its budgets."""
    a, c = problem.arrays, problem.c
    return Problem(batch=c.batch, num_layers=c.num_layers, num_q_heads=c.num_q_heads,
                   num_kv_heads=c.num_kv_heads, head_dim=c.head_dim, feat_dim=c.feat_dim,
                   dtype=problem.dtype, cu_seqlens=a["cu_seqlens"], vis_start=a["vis_start"],
                   cu_vis=a["cu_vis"], cu_keep=a["cu_vis"], softmax_scale=c.softmax_scale)


def _alloc(size, problem: Problem, device):
    """`size(problem)` bytes on the device; without that much memory free, the smaller
    workspace with which the selection does without its Gram matrices."""
    import torch

    def empty(n):
        return torch.empty(max(n, 256), dtype=torch.uint8, device=device)
    n = size(problem)
    try:
        return empty(n)
    except torch.OutOfMemoryError:
        least = size(_keep_all(problem))
        if least >= n:
            raise
        return empty(least)


def workspace(problem: Problem, device="cuda"):
    """A torch uint8 tensor of last_workspace_size bytes (torch allocations are 512-B aligned),
    or of the size without the selection's Gram matrices where the device has less free."""
    return _alloc(last_workspace_size, problem, device)


def last_scores(problem: Problem, q, k, w_out, ws, stream=None):
    p, n = _ws(ws)
    _check(load_library().last_scores(problem.ref, _ptr(q), _ptr(k), _ptr(w_out), p, n,
                                      _stream(stream)))


def last_scores_noalloc(problem: Problem, q, k, w_out, stream=None):
    """last_scores with the library's fixed scratch array instead of a workspace
    (for callers that cannot allocate device memory at run time)."""
    _check(load_library().last_scores_noalloc(problem.ref, _ptr(q), _ptr(k), _ptr(w_out),
                                              _stream(stream)))


def last_select(problem: Problem, w, x, idx_out, ws, stream=None, x_out=None):
    p, n = _ws(ws)
    _check(load_library().last_select(problem.ref, _ptr(w), _ptr(x), _ptr(idx_out), _ptr(x_out),
                                      p, n, _stream(stream)))


def last_select_topk(problem: Problem, w, idx_out, ws, stream=None, x=None, x_out=None):
    p, n = _ws(ws)
    _check(load_library().last_select_topk(problem.ref, _ptr(w), _ptr(x), _ptr(idx_out),
                                           _ptr(x_out), p, n, _stream(stream)))


class QueryRows:
    """Query rows of Table 4's attention sources: per-request offsets cu_rows
    [batch + 1] and request-local positions row_pos (host int32 arrays)."""

    def __init__(self, cu_rows: Sequence[int], row_pos: Sequence[int]):
        self.cu_rows = np.ascontiguousarray(np.asarray(cu_rows, dtype=np.int32))
        self.row_pos = np.ascontiguousarray(np.asarray(row_pos, dtype=np.int32))
        I = ctypes.POINTER(ctypes.c_int32)
        self.c_cu = self.cu_rows.ctypes.data_as(I)
        self.c_pos = self.row_pos.ctypes.data_as(I)


def last_scores_rows_workspace_size(problem: Problem, rows: QueryRows) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().last_scores_rows_workspace_size(problem.ref, rows.c_cu, rows.c_pos,
                                                          ctypes.byref(n)))
    return n.value


def rows_workspace(problem: Problem, rows: QueryRows, device="cuda"):
    import torch
    return torch.empty(max(last_scores_rows_workspace_size(problem, rows), 256), dtype=torch.uint8,
                       device=device)


def last_scores_rows(problem: Problem, rows: QueryRows, q_rows, k, w_out, ws, stream=None):
    p, n = _ws(ws)
    _check(load_library().last_scores_rows(problem.ref, rows.c_cu, rows.c_pos, _ptr(q_rows),
                                           _ptr(k), _ptr(w_out), p, n, _stream(stream)))


def last_gather(problem: Problem, x, idx, x_out, ws, stream=None):
    p, n = _ws(ws)
    _check(load_library().last_gather(problem.ref, _ptr(x), _ptr(idx), _ptr(x_out), p, n,
                                      _stream(stream)))


def last_prune(problem: Problem, q, k, x, w_out, idx_out, x_out, ws, stream=None):
    p, n = _ws(ws)
    _check(load_library().last_prune(problem.ref, _ptr(q), _ptr(k), _ptr(x), _ptr(w_out),
                                     _ptr(idx_out), _ptr(x_out), p, n, _stream(stream)))


def last_host_workspace_size(problem: Problem) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().last_host_workspace_size(problem.ref, ctypes.byref(n)))
    return n.value


def host_workspace(problem: Problem, device="cuda"):
    """A torch uint8 device tensor of last_host_workspace_size bytes, or less (see workspace)."""
    return _alloc(last_host_workspace_size, problem, device)


def last_prune_host(problem: Problem, q, k, x, w_out, idx_out, x_out, ws, stream=None):
    """last_prune on host buffers (pinned CPU tensors or numpy arrays); the copies
    are enqueued on `stream` with the path, so the outputs are ready once the
    stream has passed the call."""
    p, n = _ws(ws)
    _check(load_library().last_prune_host(problem.ref, _host_ptr(q), _host_ptr(k), _host_ptr(x),
                                          _host_ptr(w_out), _host_ptr(idx_out),
                                          _host_ptr(x_out), p, n, _stream(stream)))


def last_check_bounded_wait(ws, stream=None):
    p, _ = _ws(ws)
    _check(load_library().last_check_bounded_wait(p, _stream(stream)))


def last_poll(ws, stream=None):
    p, _ = _ws(ws)
    _check(load_library().last_poll(p, _stream(stream)))


def last_budget(n_vis: int, num: int, den: int) -> int:
    return int(load_library().last_budget(n_vis, num, den))


def last_status_string(st: int) -> str:
    return load_library().last_status_string(st).decode()


# ---- rotary positions and the key-value cache ----

_CODES, _INT32, _F32 = {}, None, None


def _dtypes():
    """torch's types, looked up once."""
    global _INT32, _F32
    import torch
    _CODES.update({torch.float32: LAST_DTYPE_F32, torch.bfloat16: LAST_DTYPE_BF16})
    _INT32, _F32 = torch.int32, torch.float32


def _code(dtype) -> int:
    if not _CODES:
        _dtypes()
    if dtype not in _CODES:
        raise ValueError(f"liblast takes float32 and bfloat16 tensors, not {dtype}")
    return _CODES[dtype]


def _int32(t, name: str, shape=None):
    """A device int32 tensor whose last dimension is contiguous."""
    if _INT32 is None:
        _dtypes()
    if t.dtype is not _INT32 or not t.is_cuda or (t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{name}: a device int32 tensor with a contiguous last dimension expected")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


class Rope:
    """Rotary positions on several axes (include/last.h `last_rotary`).  inv_freq: one frequency per
    pair; axis: the axis of each (default: all on axis 0); pairs: "half" for elements
    (i, i + rot_dim/2), "adjacent" for (2i, 2i + 1)."""

    def __init__(self, inv_freq: Sequence[float], axis: Optional[Sequence[int]] = None, pairs: str = "half",
                 num_axes: Optional[int] = None):
        self.inv_freq = np.ascontiguousarray(np.asarray(inv_freq, dtype=np.float32))
        n = len(self.inv_freq)
        self.axis = np.ascontiguousarray(np.zeros(n) if axis is None else np.asarray(axis), dtype=np.int32)
        if self.inv_freq.shape != (n,) or self.axis.shape != (n,):
            raise ValueError("inv_freq and axis must hold one value per pair")
        if num_axes is None:
            num_axes = int(self.axis.max()) + 1 if n else 1
        code = {"half": LAST_ROPE_HALF, "adjacent": LAST_ROPE_ADJACENT}[pairs]
        self.num_axes = num_axes
        self.c = _Rotary(2 * n, num_axes, code, self.inv_freq.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                         self.axis.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
        self.ref, self.addr = ctypes.byref(self.c), ctypes.addressof(self.c)

    @classmethod
    def sections(cls, sections: Sequence[int], base: float = 10000.0, pairs: str = "half"):
        """sections[a] consecutive frequencies on axis a, frequency i = base^(-2i/rot_dim)."""
        n = int(sum(sections))
        return cls(base ** (-np.arange(n, dtype=np.float64) / max(n, 1)),
                   np.repeat(np.arange(len(sections)), sections), pairs, len(sections))


class Cache:
    """A paged key-value cache (include/last.h `last_cache`) over two tensors of the caller's, k and v,
    [layers][pages][kv_heads][page_size][head_dim]; views with other strides (e.g. pages that hold
    tokens outside heads, transposed) do as well, of both tensors alike."""

    def __init__(self, k, v):
        _code(k.dtype)
        if k.dim() != 5 or v.shape != k.shape or not k.is_cuda or not v.is_cuda:
            raise ValueError("k and v: device tensors [layers][pages][kv_heads][page_size][head_dim] expected")
        if k.dtype != v.dtype or k.stride() != v.stride() or (k.shape[4] > 1 and k.stride(4) != 1):
            raise ValueError("k and v must have one dtype and the same strides, head_dim contiguous")
        self.k, self.v, self.dtype = k, v, k.dtype
        layers, pages, heads, size, dim = k.shape
        self.page_size, self.kv_heads, self.head_dim = size, heads, dim
        sl, sp, sh, st, _ = k.stride()
        self.c = _Cache(k.data_ptr(), v.data_ptr(), layers, pages, size, heads, dim, _code(k.dtype), sl, sp, sh, st)
        self.ref, self.addr = ctypes.byref(self.c), ctypes.addressof(self.c)


class Sequences:
    """Sequences of a cache (include/last.h `last_sequences`): device int32 tensors page_table
    [batch][max_pages], lens [batch] and, optionally, key_begin [batch].  Their contents may change
    between calls; a program keeps one for as long as it keeps the tensors."""

    def __init__(self, page_table, lens, key_begin=None):
        if page_table.dim() != 2:
            raise ValueError("page_table: [batch][max_pages] expected")
        b, n = page_table.shape
        self.page_table = _int32(page_table, "page_table")
        self.lens = _int32(lens, "lens", (b,))
        self.key_begin = None if key_begin is None else _int32(key_begin, "key_begin", (b,))
        self.batch = b
        self.c = _Sequences(b, n, page_table.stride(0), page_table.data_ptr(), lens.data_ptr(),
                            None if key_begin is None else key_begin.data_ptr())
        self.ref, self.addr = ctypes.byref(self.c), ctypes.addressof(self.c)


def _heads(x, out, dtype, dim, name):
    """last_heads of a [tokens][heads][dim] tensor and, optionally, its output."""
    shape, strides = x.shape, x.stride()
    if len(shape) != 3 or shape[2] != dim or x.dtype is not dtype or not x.is_cuda or (strides[2] != 1 and dim > 1):
        raise ValueError(f"{name}: a device tensor [tokens][heads][{dim}] of {dtype}, the last dimension contiguous, expected")
    if out is None:
        return _Heads(x.data_ptr(), None, shape[1], strides[0], strides[1], 0, 0)
    outs = out.stride()
    if out.shape != shape or out.dtype is not dtype or not out.is_cuda or (outs[2] != 1 and dim > 1):
        raise ValueError(f"{name}_out: a tensor like {name} expected")
    return _Heads(x.data_ptr(), out.data_ptr(), shape[1], strides[0], strides[1], outs[0], outs[1])


def _positions(positions, num_axes, tokens):
    if positions is None:
        raise ValueError("positions are required")
    if positions.dim() == 1:
        positions = positions[None]
    _int32(positions, "positions", (num_axes, tokens))
    return positions.data_ptr(), positions.stride(0) if num_axes > 1 else tokens


def _done(st) -> bool:
    """Whether the marshalling module has made the call (raises if the library refused it)."""
    if st is None:
        return False
    if st != LAST_OK:
        _check(st)
    return True


def _rope(backward, rope: Rope, positions, q, q_out, k, k_out, stream):
    if _fast is not None and _done(_fast.rope(backward, rope.addr, rope.num_axes, positions, q, q_out, k, k_out, stream)):
        return
    lib = load_library()
    call = lib.last_rope_backward if backward else lib.last_rope
    shape, dtype = q.shape, q.dtype
    t, d = shape[0], shape[-1]
    if (k is None) != (k_out is None):
        raise ValueError("k and k_out go together")
    if k is not None and k.shape[0] != t:
        raise ValueError("q and k must have the same tokens")
    qh = _heads(q, q_out, dtype, d, "q")
    kh = None if k is None else ctypes.byref(_heads(k, k_out, dtype, d, "k"))
    pos, stride = _positions(positions, rope.num_axes, t)
    _check(call(rope.ref, _code(dtype), t, d, pos, stride, ctypes.byref(qh), kh, _stream(stream)))


def last_rope(rope: Rope, positions, q, q_out, k=None, k_out=None, stream=None):
    """q and k [tokens][heads][head_dim] rotated by positions [axes][tokens] (int32) into q_out and k_out,
    which may be q and k themselves."""
    _rope(0, rope, positions, q, q_out, k, k_out, stream)


def last_rope_backward(rope: Rope, positions, q, q_out, k=None, k_out=None, stream=None):
    """The gradients q and k of the rotated heads turned back into the heads' gradients q_out and k_out."""
    _rope(1, rope, positions, q, q_out, k, k_out, stream)


def last_cache_workspace_size(cache: Cache, batch: int, num_q_heads: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().last_cache_workspace_size(cache.ref, batch, num_q_heads, ctypes.byref(n)))
    return n.value


def cache_workspace(cache: Cache, batch: int, num_q_heads: int):
    """A torch uint8 tensor of last_cache_workspace_size bytes beside the cache."""
    import torch
    return torch.empty(last_cache_workspace_size(cache, batch, num_q_heads), dtype=torch.uint8,
                       device=cache.k.device)


def last_cache_append(cache: Cache, layer: int, seqs: Sequences, k, v, ws, cu_new=None, rope: Optional[Rope] = None,
                      positions=None, q=None, q_out=None, stream=None):
    """New tokens' k and v [tokens][kv_heads][head_dim] written behind the sequences' cached ones (seqs.lens
    counts them already); with a rope, k is rotated on the way and q into q_out."""
    if _fast is not None and _done(_fast.append(
            cache.addr, layer, seqs.addr, seqs.batch, cache.head_dim, cache.dtype, k, v, ws, cu_new,
            None if rope is None else rope.addr, 0 if rope is None else rope.num_axes, positions, q, q_out, stream)):
        return
    dtype, d, t = cache.dtype, cache.head_dim, k.shape[0]
    if v.shape[0] != t or (q is not None and q.shape[0] != t):
        raise ValueError("q, k and v must have the same tokens")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    kh, vh = _heads(k, None, dtype, d, "k"), _heads(v, None, dtype, d, "v")
    qh = None if q is None else ctypes.byref(_heads(q, q_out, dtype, d, "q"))
    pos, stride = (None, 0) if rope is None else _positions(positions, rope.num_axes, t)
    p, n = _ws(ws)
    _check(load_library().last_cache_append(
        cache.ref, layer, seqs.ref, t, None if cu_new is None else _int32(cu_new, "cu_new", (seqs.batch + 1,)).data_ptr(),
        None if rope is None else rope.ref, pos, stride, qh, ctypes.byref(kh), ctypes.byref(vh), p, n, _stream(stream)))


def last_cache_attention(cache: Cache, layer: int, seqs: Sequences, q, out, ws, lse=None, softmax_scale: float = 0.0,
                         stream=None):
    """out = attention of q [batch][q_heads][head_dim] over the sequences' cached keys of one layer; lse
    [batch][q_heads] fp32 receives the log of the softmax's denominator."""
    if _fast is not None and _done(_fast.attention(cache.addr, layer, seqs.addr, seqs.batch, cache.head_dim, cache.dtype, q, out, ws,
                                                   lse, softmax_scale, stream)):
        return
    shape, d, dtype = q.shape, cache.head_dim, cache.dtype
    if len(shape) != 3 or shape[0] != seqs.batch or shape[2] != d or out.shape != shape:
        raise ValueError(f"q and out: [{seqs.batch}][q_heads][{d}] expected")
    heads, qs, os_ = shape[1], q.stride(), out.stride()
    if (q.dtype is not dtype or out.dtype is not dtype or not q.is_cuda or not out.is_cuda or qs[2] != 1 or os_[2] != 1
            or (heads > 1 and (qs[1] != d or os_[1] != d))):
        raise ValueError("q and out: device tensors of the cache's dtype, [q_heads][head_dim] contiguous, expected")
    if lse is not None and (lse.dtype is not _F32 or lse.shape != (shape[0], heads) or not lse.is_contiguous()
                            or not lse.is_cuda):
        raise ValueError("lse: a contiguous device float32 tensor [batch][q_heads] expected")
    p, n = _ws(ws)
    _check(load_library().last_cache_attention(
        cache.ref, layer, seqs.ref, heads, softmax_scale, q.data_ptr(), qs[0], out.data_ptr(), os_[0],
        None if lse is None else lse.data_ptr(), p, n, _stream(stream)))


def last_chunk_workspace_size(cache: Cache, num_q_heads: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().last_chunk_workspace_size(cache.ref, num_q_heads, ctypes.byref(n)))
    return n.value


def chunk_workspace(cache: Cache, num_q_heads: int):
    """A torch uint8 tensor of last_chunk_workspace_size bytes beside the cache."""
    import torch
    return torch.empty(last_chunk_workspace_size(cache, num_q_heads), dtype=torch.uint8, device=cache.k.device)


def _rows(x, shape, dtype, name):
    """Token stride of a device tensor [tokens][heads][width] whose tokens are contiguous."""
    s = x.stride()
    if x.shape != shape or x.dtype is not dtype or not x.is_cuda or s[2] != 1 or (shape[1] > 1 and s[1] != shape[2]):
        raise ValueError(f"{name}: a device tensor {tuple(shape)} of {dtype}, each token contiguous, expected")
    return s[0]


def _floats(x, shape, name):
    if _F32 is None:
        _dtypes()
    if x is None:
        return None
    if x.dtype is not _F32 or x.shape != shape or not x.is_contiguous() or not x.is_cuda:
        raise ValueError(f"{name}: a contiguous device float32 tensor {tuple(shape)} expected")
    return x.data_ptr()


def last_cache_chunk_attention(cache: Cache, layer: int, seqs: Sequences, q, out, ws, cu_new=None, lse=None,
                               causal: bool = True, window: int = 0, softmax_scale: float = 0.0, stream=None):
    """out = attention of the new tokens' q [tokens][q_heads][head_dim] over the sequences' cached keys of one layer (seqs.lens
    counts the new ones already); sequence b's are rows cu_new[b] .. cu_new[b+1]-1, without cu_new there is one per sequence.
    causal: up to the token's own position; window: only the last so many; lse [tokens][q_heads] fp32 receives
    the log of the softmax's denominator."""
    if _fast is not None and _done(_fast.chunk(cache.addr, layer, seqs.addr, seqs.batch, cache.head_dim, cache.dtype, q, out, ws,
                                               cu_new, lse, causal, window, softmax_scale, stream)):
        return
    d = cache.head_dim
    if q.dim() != 3 or q.shape[2] != d:
        raise ValueError(f"q: [tokens][q_heads][{d}] expected")
    t, heads = q.shape[0], q.shape[1]
    qs, os_ = _rows(q, q.shape, cache.dtype, "q"), _rows(out, q.shape, cache.dtype, "out")
    p, n = _ws(ws)
    _check(load_library().last_cache_chunk_attention(
        cache.ref, layer, seqs.ref, t, None if cu_new is None else _int32(cu_new, "cu_new", (seqs.batch + 1,)).data_ptr(), heads,
        softmax_scale, int(causal), window, q.data_ptr(), qs, out.data_ptr(), os_, _floats(lse, (t, heads), "lse"), p, n,
        _stream(stream)))


def last_cache_diff_attention(cache: Cache, layer: int, seqs: Sequences, q, out, ws, lam, cu_new=None, norm_weight=None,
                              norm_eps: float = 1e-5, out_scale: float = 1.0, causal: bool = True, window: int = 0,
                              softmax_scale: float = 0.0, stream=None):
    """Differential attention of the new tokens' q [tokens][q_heads][head_dim], heads in pairs, over a cache whose K and V heads
    are paired too: out [tokens][q_heads / 2][2 head_dim] = softmax map 1 - lam[pair] x map 2, with norm_weight
    [2 head_dim] RMS-normalised, times out_scale.  lam [q_heads / 2] and norm_weight: fp32.  The rest is as for
    last_cache_chunk_attention."""
    if _fast is not None and _done(_fast.difference(cache.addr, layer, seqs.addr, seqs.batch, cache.head_dim, cache.dtype, q, out, ws,
                                                    cu_new, lam, norm_weight, norm_eps, out_scale, causal, window, softmax_scale, stream)):
        return
    d = cache.head_dim
    if q.dim() != 3 or q.shape[2] != d or q.shape[1] % 2 != 0:
        raise ValueError(f"q: [tokens][q_heads][{d}], an even number of heads, expected")
    t, heads = q.shape[0], q.shape[1]
    qs, os_ = _rows(q, q.shape, cache.dtype, "q"), _rows(out, (t, heads // 2, 2 * d), cache.dtype, "out")
    if lam is None:
        raise ValueError("lam is required")
    diff = _Difference(_floats(lam, (heads // 2,), "lam"), _floats(norm_weight, (2 * d,), "norm_weight"), norm_eps, out_scale)
    p, n = _ws(ws)
    _check(load_library().last_cache_diff_attention(
        cache.ref, layer, seqs.ref, t, None if cu_new is None else _int32(cu_new, "cu_new", (seqs.batch + 1,)).data_ptr(), heads,
        softmax_scale, int(causal), window, ctypes.byref(diff), q.data_ptr(), qs, out.data_ptr(), os_, p, n, _stream(stream)))


def last_cache_copy(cache: Cache, src, dst, ws, stream=None):
    """Pages src[i] copied to pages dst[i] (device int32), every layer, K and V."""
    if _fast is not None and _done(_fast.copy(cache.addr, src, dst, ws, stream)):
        return
    n = src.shape[0]
    p, nb = _ws(ws)
    _check(load_library().last_cache_copy(cache.ref, n, _int32(src, "src", (n,)).data_ptr(),
                                          _int32(dst, "dst", (n,)).data_ptr(), p, nb, _stream(stream)))


def last_cache_compact(cache: Cache, seqs: Sequences, dst_table, cu_keep, idx, lens_out, ws, span_begin=None,
                       span_len=None, stream=None):
    """The sequences' tokens outside their spans and the spans' tokens idx (as last_select writes them),
    in order, copied to the pages of dst_table [batch][max_pages]; lens_out [batch] receives the new lengths."""
    if _fast is not None and _done(_fast.compact(cache.addr, seqs.addr, seqs.batch, dst_table, cu_keep, idx, lens_out, ws, span_begin,
                                                 span_len, stream)):
        return
    b, shape = seqs.batch, dst_table.shape
    if len(shape) != 2 or shape[0] != b or idx.dim() != 1:
        raise ValueError("dst_table: [batch][max_pages], idx: one dimension expected")

    def per_sequence(t, name):
        return None if t is None else _int32(t, name, (b,)).data_ptr()
    p, n = _ws(ws)
    _check(load_library().last_cache_compact(
        cache.ref, seqs.ref, _int32(dst_table, "dst_table").data_ptr(), shape[1], dst_table.stride(0),
        per_sequence(span_begin, "span_begin"), per_sequence(span_len, "span_len"),
        _int32(cu_keep, "cu_keep", (b + 1,)).data_ptr(), _int32(idx, "idx").data_ptr(), idx.shape[0],
        per_sequence(lens_out, "lens_out"), p, n, _stream(stream)))


class PagePool:
    """Who holds which page of a cache (include/last.h `last_page_pool`), in host memory."""

    def __init__(self, num_pages: int):
        self.holders = np.zeros(max(num_pages, 1), dtype=np.int32)
        self.free_pages = np.zeros(max(num_pages, 1), dtype=np.int32)
        I = ctypes.POINTER(ctypes.c_int32)
        self.c = _PagePool(num_pages, 0, self.holders.ctypes.data_as(I), self.free_pages.ctypes.data_as(I))
        last_pages_init(self)

    @property
    def num_free(self) -> int:
        return self.c.num_free


def _page_list(pages):
    a = np.ascontiguousarray(np.asarray(pages, dtype=np.int32).reshape(-1))
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def last_pages_init(pool: PagePool):
    _check(load_library().last_pages_init(ctypes.byref(pool.c)))


def last_pages_take(pool: PagePool, n: int) -> np.ndarray:
    """n free pages, one holder each."""
    a, ptr = _page_list(np.zeros(max(n, 0)))
    _check(load_library().last_pages_take(ctypes.byref(pool.c), n, ptr))
    return a


def last_pages_share(pool: PagePool, pages):
    a, ptr = _page_list(pages)
    _check(load_library().last_pages_share(ctypes.byref(pool.c), len(a), ptr))


def last_pages_release(pool: PagePool, pages):
    a, ptr = _page_list(pages)
    _check(load_library().last_pages_release(ctypes.byref(pool.c), len(a), ptr))
