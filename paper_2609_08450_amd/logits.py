"""Penalties, biases and grammar masks on logits, as the FP32 rows that a ``topk`` selects from::

    rows = logits.adjust(x, tokens=tokens, token_starts=starts, repetition=rep, mask=mask, row_mask=state)
    idx, val = select(rows, offsets, lengths)          # a topk.TopK, of a row's vocabulary

``adjust`` forwards to serve_adjust() (include/serve_step.h, which has the contract): on ``stream`` or the
current one, without a synchronisation or a fallback; errors are ``paged.PagedError``.
"""
from __future__ import annotations

import ctypes

import torch

from . import _serve
from . import paged as _paged
from . import topk as _topk

PagedError = _paged.PagedError


def _rows(t, dtypes, shape, name, dev):
    if t.get_device() != dev:
        raise _paged._elsewhere(t, dev, name)
    if t.dtype not in dtypes or (shape is not None and t.shape != shape) or t.dim() != 2:
        raise PagedError(f"{name} must be {' or '.join(map(str, dtypes))} of shape "
                         f"{tuple(shape) if shape is not None else '(rows, vocab)'}, got {t.dtype} {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1 and t.numel():
        raise PagedError(f"{name} must have a contiguous last axis")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1]


def adjust(x, out=None, *, tokens=None, token_starts=None, prompt_lens=None, repetition=None, frequency=None,
           presence=None, bias_ids=None, bias=None, bias_starts=None, mask=None, row_mask=None, stream=None):
    """Forwards to serve_adjust(): ``x`` [rows, vocab] of bfloat16, float16 or float32 to ``out`` float32, which may
    be x itself.

    tokens, token_starts     int32 [any], int64 [rows + 1]: each row's tokens so far, the first
    prompt_lens              (int32 [rows]) of which are the prompt's;
    repetition, frequency, presence   float32 [rows];
    bias_ids, bias, bias_starts       int32 and float32 [any], int64 [rows + 1];
    mask, row_mask           int32 [masks, words] of bits, token t's bit t % 32 of word t // 32 set where it is
                             allowed; int32 [rows]: each row's mask, negative for none (None: row i's is mask i).

    Returns out."""
    dev = _paged._device(x, "x")
    xp, x_row = _rows(x, _serve.ACTS, None, "x", dev)
    rows, vocab = x.shape
    if out is None:
        out = _serve.empty(x.shape, x, torch.float32, stream)
    op, out_row = _rows(out, (torch.float32,), x.shape, "out", dev)
    if rows > 1 and out_row < vocab:
        raise PagedError("out's rows must not overlap")

    def vec(t, dtype, n, name):
        return None if t is None else _paged._vec(t, dtype, t.numel() if n is None else n, name, dev)

    if (tokens is None) != (token_starts is None):
        raise PagedError("tokens and token_starts belong together")
    if tokens is None and any(t is not None for t in (prompt_lens, repetition, frequency, presence)):
        raise PagedError("penalties need tokens")
    if not (bias_ids is None) == (bias is None) == (bias_starts is None):
        raise PagedError("bias_ids, bias and bias_starts belong together")
    if bias is not None and bias.numel() != bias_ids.numel():
        raise PagedError("bias_ids and bias must have one length")
    if row_mask is not None and mask is None:
        raise PagedError("row_mask belongs to a mask")
    mp, stride, masks = None, 0, 0
    if mask is not None:
        mp, stride = _rows(mask, (torch.int32,), None, "mask", dev)
        masks, words = mask.shape
        if words * 32 < vocab:
            raise PagedError(f"mask must have {(vocab + 31) // 32} words, got {words}")
        if row_mask is None and masks != rows:
            raise PagedError(f"{masks} masks for {rows} rows need a row_mask")
    i32, i64, f32 = torch.int32, torch.int64, torch.float32
    # an empty list has no address, and is none
    lists = _serve.Lists(vec(tokens, i32, None, "tokens"), vec(token_starts, i64, rows + 1, "token_starts"),
                         vec(prompt_lens, i32, rows, "prompt_lens"), vec(repetition, f32, rows, "repetition"),
                         vec(frequency, f32, rows, "frequency"), vec(presence, f32, rows, "presence"),
                         vec(bias_ids, i32, None, "bias_ids"), vec(bias, f32, None, "bias"),
                         vec(bias_starts, i64, rows + 1, "bias_starts"), mp, stride, masks,
                         vec(row_mask, i32, rows, "row_mask"))
    _serve.check((_serve._lib or _serve.lib()).serve_adjust(
        _serve.ACTS[x.dtype], xp, x_row, op, out_row, rows, vocab, ctypes.byref(lists), _topk._stream(stream)),
        "serve_adjust")
    return out
