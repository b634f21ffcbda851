"""Eviction from a paged cache by accumulated attention weight.

Each row of weights has the layout that ``topk`` selects from: FP32, one for every token of a
request, at an offset of the request's own::

    out = paged.attend(cache, q, table, row_starts, row_lengths, scale, lse=lse)
    evict.weigh(cache, q, lse, table, row_starts, row_lengths, scale, weights, offsets)
    ...                                     # and where a request has grown too long:
    idx, _ = select(weights, offsets + first, (lens - first - last).clamp(min=0))   # a topk.TopK
    evict.keep(idx, lens, first, last, kept, counts, base=first, weights=weights, weight_offsets=offsets)
    evict.compact(cache, table, kept, counts)
    paged.tables(ring, pool, lens, counts - lens, table, ...)     # takes the free pages back

The functions forward to serve_weigh(), serve_keep() and serve_compact() (include/serve_step.h, which
has the contract of each), as those of ``paged`` do: on ``stream`` or the current one, without a
synchronisation or a fallback; errors are ``paged.PagedError``.
"""
from __future__ import annotations

import torch

from . import _serve
from . import paged as _paged
from . import topk as _topk

PagedError = _paged.PagedError


NO_WORKSPACE = 256  # bytes that stand for none
_sizes = {}  # bytes by (rows, requests, heads, cache heads)


def workspace_size(cache, n_rows: int, n_requests: int, heads: int) -> int:
    key = (n_rows, n_requests, heads, cache.n_heads)
    size = _sizes.get(key)
    if size is None:
        size = _serve.lib().serve_weigh_workspace(*key)
        if size == 0:
            raise PagedError("serve_weigh_workspace: invalid arguments or device")
        if len(_sizes) >= 1024:
            _sizes.clear()
        _sizes[key] = size
    return size


def weigh(cache, q, lse, table, row_starts, row_lengths, scale: float, weights, weight_offsets, workspace=None,
          stream=None) -> None:
    """Forwards to serve_weigh(): adds to each request's weights (any contiguous float32 tensor, request r's
    from weight_offsets[r] on) what its tokens got of the attention of q [rows, heads, dim], whose ``lse``
    float32 [rows, heads] ``paged.attend`` gave.  The launch is laid out for the table's width: where a program knows that
    requests are far shorter, ``table[:, :pages]`` is faster.  ``workspace``: uint8 of ``workspace_size`` bytes, for a
    program that keeps one; where that is 256 (single tokens, few rows) a call uses none."""
    dev = cache._on_current()
    qp, q_row, q_head = _paged._rows3(q, None, cache.head_dim, "q", dev)
    rows, heads, _ = q.shape
    at, stride, width = _paged._table(table, dev)
    n = table.shape[0]
    wp = size = 0
    if workspace is not None:
        if workspace.get_device() != dev:
            raise _paged._elsewhere(workspace, dev, "workspace")
        if workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
            raise PagedError("workspace must be a contiguous device tensor of uint8")
        wp, size = workspace.data_ptr(), workspace.numel()
    elif rows > n:
        size = workspace_size(cache, rows, n, heads)
        if size > NO_WORKSPACE:
            workspace = _serve.empty(size, q, torch.uint8, stream)
            wp = workspace.data_ptr()
    _serve.check((_serve._lib or _serve.lib()).serve_weigh(
        cache._ref, _paged.ACTS[q.dtype], qp, q_row, q_head, heads,
        _serve.flat(lse, torch.float32, (rows, heads), "lse", dev), at, stride, width,
        _serve.vec(row_starts, torch.int32, n + 1, "row_starts", dev), n,
        _serve.vec(row_lengths, torch.int32, rows, "row_lengths", dev), rows, scale,
        _serve.flat(weights, torch.float32, None, "weights", dev),
        _serve.vec(weight_offsets, torch.int64, n, "weight_offsets", dev), wp, size, _topk._stream(stream)),
        "serve_weigh")


def keep(idx, lens, first: int, last: int, kept, counts, *, base: int = 0, weights=None, weight_offsets=None,
         stream=None) -> None:
    """Forwards to serve_keep(): of each request's ``lens[r]`` tokens the first ``first``, the last ``last`` and
    ``base + idx[r]`` (int32 [requests, K], a selection's indices) stay.  Writes their numbers to ``kept`` int32
    [requests, width], width >= first + K + last, ascending and then -1, and how many they are to ``counts``;
    moves their ``weights`` along, where given."""
    dev = _paged._device(idx, "idx")
    i32 = torch.int32
    n = lens.numel()
    at = _paged._ptr(idx, i32, (n, None), "idx", dev)
    if (weights is None) != (weight_offsets is None):
        raise PagedError("weights and weight_offsets belong together")
    wp, op = None, None
    if weights is not None:
        wp = _serve.flat(weights, torch.float32, None, "weights", dev)
        op = _serve.vec(weight_offsets, torch.int64, n, "weight_offsets", dev)
    _serve.check((_serve._lib or _serve.lib()).serve_keep(
        at, idx.shape[1], base, _serve.vec(lens, i32, n, "lens", dev), n, first, last,
        _paged._ptr(kept, i32, (n, None), "kept", dev), kept.shape[1], _serve.vec(counts, i32, n, "counts", dev), wp, op,
        _topk._stream(stream)), "serve_keep")


def compact(cache, table, kept, counts, stream=None) -> None:
    """Forwards to serve_compact(): token i of request r becomes what its token kept[r][i] was, in place, for
    i < counts[r].  The pages behind are free then: ``paged.tables`` takes them back."""
    dev = cache._on_current()
    at, stride, width = _paged._table(table, dev)
    n = table.shape[0]
    kp = _paged._ptr(kept, torch.int32, (n, None), "kept", dev)
    _serve.check((_serve._lib or _serve.lib()).serve_compact(
        cache._ref, at, stride, width, kp, kept.shape[1], _serve.vec(counts, torch.int32, n, "counts", dev), n,
        _topk._stream(stream)), "serve_compact")
