"""Python binding of the paged_kv C-ABI: a paged 8-bit cache and what reads it.

The calls around a selection, in the order of a serving step::

    tables -> store -> score -> topk.topk_ragged -> attend_selected
                    -> attend                      (layers that read everything)

As in ``topk``, every function checks and marshals arguments and forwards
device pointers and the stream to the library (libpaged_kv.so); all work runs
in its HIP kernels, there is no fallback.  include/paged_kv.h holds the
contract of each call.

``stream`` (a torch stream or a handle; None: the current one) is where a call
runs.  Inputs have to be ready there, and an output that a call makes belongs to
that stream, as if torch had made it there.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import topk as _topk
from .build import PAGED_LIB_PATH

CODES = {torch.float8_e4m3fn: 0, torch.int8: 1}
ACTS = {torch.bfloat16: 0, torch.float16: 1}
WORKSPACE_ZEROED = 8192


class PagedError(RuntimeError):
    pass


class _Cache(ctypes.Structure):
    """Mirror of paged_kv_cache (include/paged_kv.h)."""

    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("page_stride", ctypes.c_int64),
        ("scale_stride", ctypes.c_int64),
        ("n_pages", ctypes.c_int32),
        ("page", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("code", ctypes.c_int32),
    ]


_lib = None


def lib():
    """Loads libpaged_kv.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(PAGED_LIB_PATH):
            raise PagedError(f"{PAGED_LIB_PATH} is missing: build it with "
                             "`python -m paper_2609_08450_amd.build` (no CPU fallback exists)")
        L = ctypes.CDLL(PAGED_LIB_PATH)
        _topk._check_single_hip_runtime()
        P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        C, size = ctypes.POINTER(_Cache), ctypes.c_size_t
        L.paged_kv_tables.argtypes = [P, i32, P, P, P, P, P, i32, P, i32, i32, i32, i32, P, P, P, P, P]
        L.paged_kv_store.argtypes = [C, i32, P, i64, i64, P, i64, i64, P, i32, P]
        L.paged_kv_attend_workspace.argtypes = [i32, i32, i32, i32, i32]
        L.paged_kv_attend_workspace.restype = size
        L.paged_kv_attend.argtypes = [C, i32, P, i64, i64, i32, P, i32, i32, P, i32, P, i32, f32, P, P,
                                      P, size, P]
        L.paged_kv_attend_selected.argtypes = [C, i32, P, i64, i64, i32, P, i32, P, i32, i32, P, i32, P,
                                               i32, f32, P, P, P, size, P]
        L.paged_kv_score.argtypes = [C, i32, P, i64, i64, i32, P, P, i32, i32, P, i32, P, i32, f32, P, P, P]
        for name in ("tables", "store", "attend", "attend_selected", "score"):
            getattr(L, "paged_kv_" + name).restype = ctypes.c_int
        L.paged_kv_status_str.argtypes = [ctypes.c_int]
        L.paged_kv_status_str.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc: int, what: str):
    if rc != 0:
        raise PagedError(f"{what} failed: {lib().paged_kv_status_str(rc).decode()} ({rc})")


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device(t, name):
    """The device of a call: its first tensor's, which has to be the current one (launches go there)."""
    dev = t.get_device()
    if dev < 0:
        raise PagedError(f"{name} must be a device tensor")
    if dev != _current_device():
        raise PagedError(f"{name} is on cuda:{dev}, but the current device is cuda:{_current_device()}")
    return dev


def _elsewhere(t, dev, name):
    if t.get_device() < 0:
        return PagedError(f"{name} must be a device tensor")
    return PagedError(f"{name} is on cuda:{t.get_device()}, the call's other tensors are on cuda:{dev}")


def _ptr(t, dtype, shape, name, dev):
    """Address of a contiguous tensor of this type and shape (None: any size) on device `dev`."""
    if t.get_device() != dev:
        raise _elsewhere(t, dev, name)
    if t.dtype is not dtype:
        raise PagedError(f"{name} must be {dtype}, got {t.dtype}")
    got = t.shape
    if len(got) != len(shape) or any(b is not None and a != b for a, b in zip(got, shape)):
        raise PagedError(f"{name} must have shape {tuple(shape)}, got {tuple(got)}")
    if not t.is_contiguous():
        raise PagedError(f"{name} must be contiguous")
    return t.data_ptr()


def _vec(t, dtype, n, name, dev):
    """_ptr of a tensor with one axis, in fewer steps: the short calls' host time counts."""
    if t.dtype is dtype and t.get_device() == dev and t.numel() == n and t.dim() == 1 and t.is_contiguous():
        return t.data_ptr()
    return _ptr(t, dtype, (n,), name, dev)


def _rows3(t, heads, dim, name, dev):
    """Address and strides of activations [rows, heads, dim] whose last axis is contiguous."""
    if t.get_device() != dev:
        raise _elsewhere(t, dev, name)
    if t.dtype not in ACTS:
        raise PagedError(f"{name} must be bfloat16 or float16, got {t.dtype}")
    if t.dim() != 3 or t.shape[2] != dim or (heads is not None and t.shape[1] != heads):
        raise PagedError(f"{name} must have shape (rows, {heads or 'heads'}, {dim}), got {tuple(t.shape)}")
    row, head, last = t.stride()
    if t.shape[0] == 1:
        row = 0
    if t.shape[1] == 1:
        head = 0
    if t.numel() and (last != 1 or row % 8 or head % 8 or t.data_ptr() % 16):
        raise PagedError(f"{name} must have a contiguous last axis, strides that are multiples of 8 "
                         "elements and a 16-byte aligned address")
    return t.data_ptr(), row, head


def _table(table, dev, n=None):
    """Address, stride and width of a block table [requests, width], its last axis contiguous."""
    if table.get_device() != dev:
        raise _elsewhere(table, dev, "table")
    if table.dtype is not torch.int32 or table.dim() != 2:
        raise PagedError("table must be a device tensor of int32 [requests, width]")
    if n is not None and table.shape[0] != n:
        raise PagedError(f"table must have {n} rows, got {table.shape[0]}")
    width = table.shape[1]
    stride = table.stride(0) if table.shape[0] > 1 else width
    if table.numel() and (table.stride(1) != 1 and width > 1 or stride < width):
        raise PagedError("table must have a contiguous last axis")
    return table.data_ptr(), stride, width


def _on(stream):
    """The context in which torch allocates and works on `stream` (a handle too; None: the current one)."""
    if stream is not None and not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_topk._stream(stream))
    return torch.cuda.stream(stream)


class PagedCache:
    """Pages of keys (and values) in 8 bits with their scales, and the workspace of
    the attention calls on them.

    ``k``, ``v`` [n_pages, n_heads, page, head_dim] of float8_e4m3fn or int8;
    ``k_scale``, ``v_scale`` float32 [n_pages, n_heads].  Pages may be strided
    along the first axis (a layer's slice of [n_pages, layers, ...]).  Calls
    that overlap on different streams each need a workspace of their own
    (``workspace=``, from ``alloc_workspace``).  A workspace that a larger one
    replaces stays allocated as long as the cache: graphs that were captured
    with it remain valid.  A captured call needs one of its size already: from a
    call before the capture, or its own.
    """

    def __init__(self, n_pages: int, page: int, n_heads: int, head_dim: int,
                 dtype=torch.float8_e4m3fn, values: bool = True, device="cuda"):
        if dtype not in CODES:
            raise PagedError(f"a cache holds float8_e4m3fn or int8, got {dtype}")

        def side():
            codes = torch.zeros((n_pages, n_heads, page, head_dim), dtype=torch.uint8, device=device)
            return codes.view(dtype), torch.ones((n_pages, n_heads), device=device)

        self._set(*side(), *(side() if values else (None, None)))

    @classmethod
    def of(cls, k, k_scale, v=None, v_scale=None) -> "PagedCache":
        """A cache on tensors that the program has allocated."""
        self = cls.__new__(cls)
        self._set(k, k_scale, v, v_scale)
        return self

    def _set(self, k, k_scale, v, v_scale):
        if (v is None) != (v_scale is None):
            raise PagedError("v and v_scale belong together")
        for codes, scale, name in ((k, k_scale, "k"), (v, v_scale, "v")):
            if codes is None:
                continue
            if not codes.is_cuda or scale.get_device() != k.get_device() or codes.get_device() != k.get_device():
                raise PagedError(f"{name} and its scale must be device tensors, on one device")
            if codes.dtype not in CODES:
                raise PagedError(f"{name} must be float8_e4m3fn or int8, got {codes.dtype}")
            if codes.dim() != 4 or not codes[:1].is_contiguous():
                raise PagedError(f"{name} must be [pages, heads, page, dim], contiguous within a page")
            if scale.dtype is not torch.float32 or scale.shape != codes.shape[:2] or scale.stride(1) != 1:
                raise PagedError(f"{name}_scale must be float32 [pages, heads], contiguous within a page")
        if v is not None and (v.shape != k.shape or v.dtype != k.dtype or v.stride() != k.stride()
                              or v_scale.stride() != k_scale.stride()):
            raise PagedError("k and v must have one shape, type and layout")
        self.k, self.k_scale, self.v, self.v_scale = k, k_scale, v, v_scale
        self.n_pages, self.n_heads, self.page, self.head_dim = k.shape
        one = self.n_pages == 1  # the stride of an axis of length one says nothing
        self._c = _Cache(k.data_ptr(), v.data_ptr() if v is not None else None, k_scale.data_ptr(),
                         v_scale.data_ptr() if v is not None else None,
                         self.n_heads * self.page * self.head_dim if one else k.stride(0),
                         self.n_heads if one else k_scale.stride(0),
                         self.n_pages, self.page, self.n_heads, self.head_dim, CODES[k.dtype])
        self._ref = ctypes.byref(self._c)
        self._device = k.get_device()
        self._sizes = {}
        self.workspace, self._replaced = None, []

    def workspace_size(self, n_rows: int, n_requests: int, heads: int) -> int:
        key = (n_rows, n_requests, heads)
        size = self._sizes.get(key)
        if size is None:
            size = lib().paged_kv_attend_workspace(n_rows, n_requests, heads, self.n_heads, self.head_dim)
            if size == 0:
                raise PagedError("paged_kv_attend_workspace: invalid arguments or device")
            if len(self._sizes) >= 1024:
                self._sizes.clear()
            self._sizes[key] = size
        return size

    def alloc_workspace(self, n_rows: int, n_requests: int, heads: int, stream=None) -> torch.Tensor:
        """A workspace for attention calls of these sizes, ready for its first use on `stream`."""
        return self._ready(self.workspace_size(n_rows, n_requests, heads), stream)

    def _ready(self, size, stream, captured=True):
        with _on(stream):
            if not captured and torch.cuda.is_current_stream_capturing():
                raise PagedError("a cache makes its workspace outside of a capture: make a call of these sizes "
                                 "before it, or pass workspace=")
            ws = torch.empty(size, dtype=torch.uint8, device=self.k.device)
            ws[:WORKSPACE_ZEROED].zero_()
        return ws

    def _on_current(self):
        """The device of the cache, which has to be the current one (launches go there)."""
        if self._device != _current_device():
            raise PagedError(f"the cache is on cuda:{self._device}, but the current device is cuda:{_current_device()}")
        return self._device

    def _space(self, workspace, n_rows, n_requests, heads, stream):
        need = self.workspace_size(n_rows, n_requests, heads)
        if workspace is None:
            if self.workspace is None or self.workspace.numel() < need:
                # A captured graph, or a kernel on another stream, may still use the one
                # that is replaced, so it stays.  The new one has room to spare (an eighth
                # more), so that growing sizes replace it seldom.  None is made under
                # capture: it would be the graph's memory, and zeroed by the replays alone.
                made = self._ready(need + max(need // 8, 1 << 20), stream, captured=False)
                if self.workspace is not None:
                    self._replaced.append(self.workspace)
                self.workspace = made
            workspace = self.workspace
        elif workspace.get_device() != self._device:
            raise _elsewhere(workspace, self._device, "workspace")
        elif workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
            raise PagedError("workspace must be a contiguous device tensor of uint8")
        return workspace.data_ptr(), workspace.numel()


def tables(ring, pool, lens, new_lens, table, page: int, *, pool_out, lens_out, row_starts, row_request,
           row_lengths, slots, stream=None) -> None:
    """Forwards to paged_kv_tables(): a step's block tables, rows and slots from
    request lengths.  ``pool`` int32 [4] (place of the ring's first free page,
    count, ...); the number of rows is that of ``slots``.  ``pool_out`` may be
    ``pool``; ``lens_out`` is another tensor than ``lens``."""
    n, rows = lens.numel(), slots.numel()
    i32 = torch.int32
    dev = _device(table, "table")
    at, stride, width = _table(table, dev, n)
    _check((_lib or lib()).paged_kv_tables(
        _ptr(ring, i32, (None,), "ring", dev), ring.numel(), _vec(pool, i32, 4, "pool", dev),
        _vec(pool_out, i32, 4, "pool_out", dev), _vec(lens, i32, n, "lens", dev), _vec(new_lens, i32, n, "new_lens", dev),
        _vec(lens_out, i32, n, "lens_out", dev), n, at, stride, width, page, rows,
        _vec(row_starts, i32, n + 1, "row_starts", dev), _vec(row_request, i32, rows, "row_request", dev),
        _vec(row_lengths, i32, rows, "row_lengths", dev), _vec(slots, torch.int64, rows, "slots", dev),
        _topk._stream(stream)), "paged_kv_tables")


def store(cache: PagedCache, k_new, v_new, slots, stream=None) -> None:
    """Forwards to paged_kv_store(): new entries [rows, heads, dim] into the pages."""
    dev = cache._on_current()
    k, k_row, k_head = _rows3(k_new, cache.n_heads, cache.head_dim, "k_new", dev)
    n = k_new.shape[0]
    v, v_row, v_head = None, 0, 0
    if v_new is not None:
        v, v_row, v_head = _rows3(v_new, cache.n_heads, cache.head_dim, "v_new", dev)
        if v_new.shape[0] != n or v_new.dtype is not k_new.dtype:
            raise PagedError("k_new and v_new must have one type and number of rows")
    if (v_new is None) != (cache.v is None):
        raise PagedError("v_new belongs to a cache with values, and to no other")
    _check((_lib or lib()).paged_kv_store(cache._ref, ACTS[k_new.dtype], k, k_row, k_head, v, v_row, v_head,
                                          _vec(slots, torch.int64, n, "slots", dev), n, _topk._stream(stream)),
           "paged_kv_store")


def _outputs(q, out, lse, stream, dev):
    if out is None and stream is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif out is None:  # of the stream that writes it: its memory may still be in use on the current one
        with _on(stream):
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    at = _ptr(out, q.dtype, q.shape, "out", dev)
    return out, at, _ptr(lse, torch.float32, q.shape[:2], "lse", dev) if lse is not None else None


def attend(cache: PagedCache, q, table, row_starts, row_lengths, scale: float, out=None, lse=None,
           workspace=None, stream=None):
    """Forwards to paged_kv_attend(): each row of q [rows, heads, dim] over the
    first row_lengths[i] tokens of its request.  Returns out."""
    dev = cache._on_current()
    qp, q_row, q_head = _rows3(q, None, cache.head_dim, "q", dev)
    rows, heads, _ = q.shape
    at, stride, width = _table(table, dev)
    n = table.shape[0]
    out, op, lp = _outputs(q, out, lse, stream, dev)
    ws, size = cache._space(workspace, rows, n, heads, stream)
    _check((_lib or lib()).paged_kv_attend(
        cache._ref, ACTS[q.dtype], qp, q_row, q_head, heads, at, stride, width,
        _vec(row_starts, torch.int32, n + 1, "row_starts", dev), n,
        _vec(row_lengths, torch.int32, rows, "row_lengths", dev), rows, scale, op, lp, ws, size,
        _topk._stream(stream)), "paged_kv_attend")
    return out


def attend_selected(cache: PagedCache, q, idx, table, row_request, row_lengths, scale: float, out=None, lse=None,
                    workspace=None, stream=None):
    """Forwards to paged_kv_attend_selected(): each row of q over the tokens
    idx[i] of its request (a selection's out_idx).  Returns out."""
    dev = cache._on_current()
    qp, q_row, q_head = _rows3(q, None, cache.head_dim, "q", dev)
    rows, heads, _ = q.shape
    at, stride, width = _table(table, dev)
    n = table.shape[0]
    out, op, lp = _outputs(q, out, lse, stream, dev)
    ws, size = cache._space(workspace, rows, n, heads, stream)
    _check((_lib or lib()).paged_kv_attend_selected(
        cache._ref, ACTS[q.dtype], qp, q_row, q_head, heads, _ptr(idx, torch.int32, (rows, None), "idx", dev),
        idx.shape[1], at, stride, width, _vec(row_request, torch.int32, rows, "row_request", dev), n,
        _vec(row_lengths, torch.int32, rows, "row_lengths", dev), rows, scale, op, lp, ws, size,
        _topk._stream(stream)), "paged_kv_attend_selected")
    return out


def score(cache: PagedCache, q, w, table, row_request, row_lengths, scale: float, scores, row_offsets,
          stream=None) -> None:
    """Forwards to paged_kv_score(): row i's scores of its visible tokens to
    scores[row_offsets[i] ..] (any contiguous float32 tensor), as topk_ragged reads them."""
    dev = cache._on_current()
    qp, q_row, q_head = _rows3(q, None, cache.head_dim, "q", dev)
    rows, heads, _ = q.shape
    at, stride, width = _table(table, dev)
    _check((_lib or lib()).paged_kv_score(
        cache._ref, ACTS[q.dtype], qp, q_row, q_head, heads, _ptr(w, torch.float32, (rows, heads), "w", dev), at, stride,
        width, _vec(row_request, torch.int32, rows, "row_request", dev), table.shape[0],
        _vec(row_lengths, torch.int32, rows, "row_lengths", dev), rows, scale,
        _ptr(scores, torch.float32, scores.shape, "scores", dev), _vec(row_offsets, torch.int64, rows, "row_offsets", dev),
        _topk._stream(stream)), "paged_kv_score")
