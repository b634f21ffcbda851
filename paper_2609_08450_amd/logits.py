"""Penalties, biases and grammar masks on logits, as the FP32 rows that a ``topk`` selects from::

    rows = logits.adjust(x, tokens=tokens, token_starts=starts, repetition=rep, mask=mask, row_mask=state)
    idx, val = select(rows, offsets, lengths)          # a topk.TopK, of a row's vocabulary

``adjust`` forwards to serve_adjust() (include/serve_step.h, which has the contract): on ``stream`` or the
current one, without a synchronisation or a fallback; errors are ``paged.PagedError``.
"""
from __future__ import annotations

import torch

from . import _serve
from . import paged as _paged
from . import topk as _topk

PagedError = _paged.PagedError


def _rows(t, ok, shape, what, name, dev):
    """Address and row stride of a tensor [rows, columns] whose last axis is contiguous."""
    got, at = t.shape, t.stride()
    if t.get_device() != dev:
        raise _paged._elsewhere(t, dev, name)
    if not ok or len(got) != 2 or (shape is not None and got != shape):
        raise PagedError(f"{name} must be {what}, got {t.dtype} {tuple(got)}")
    if at[1] != 1 and got[1] > 1 and got[0]:
        raise PagedError(f"{name} must have a contiguous last axis")
    return t.data_ptr(), at[0] if got[0] > 1 else got[1]


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
    act, i32, i64, f32 = _serve.ACTS.get(x.dtype), torch.int32, torch.int64, torch.float32
    xp, x_row = _rows(x, act is not None, None, "bfloat16, float16 or float32 [rows, vocab]", "x", dev)
    rows, vocab = shape = x.shape
    if out is None:
        out = _serve.empty(shape, x, f32, stream)
    op, out_row = _rows(out, out.dtype is f32, shape, f"float32 of shape {tuple(shape)}", "out", dev)
    if rows > 1 and out_row < vocab:
        raise PagedError("out's rows must not overlap")
    vec = _serve.vec

    if (tokens is None) != (token_starts is None):
        raise PagedError("tokens and token_starts belong together")
    if tokens is None and any(t is not None for t in (prompt_lens, repetition, frequency, presence)):
        raise PagedError("penalties need tokens")
    if not (bias_ids is None) == (bias is None) == (bias_starts is None):
        raise PagedError("bias_ids, bias and bias_starts belong together")
    if row_mask is not None and mask is None:
        raise PagedError("row_mask belongs to a mask")
    mp = stride = masks = 0
    if mask is not None:
        mp, stride = _rows(mask, mask.dtype is i32, None, "int32 [masks, words]", "mask", dev)
        masks, words = mask.shape
        if words * 32 < vocab:
            raise PagedError(f"mask must have {(vocab + 31) // 32} words, got {words}")
        if row_mask is None and masks != rows:
            raise PagedError(f"{masks} masks for {rows} rows need a row_mask")
    # (an empty list has no address, and is none)
    lists = _serve.pack_lists(
        0 if tokens is None else vec(tokens, i32, None, "tokens", dev),
        0 if tokens is None else vec(token_starts, i64, rows + 1, "token_starts", dev),
        0 if prompt_lens is None else vec(prompt_lens, i32, rows, "prompt_lens", dev),
        0 if repetition is None else vec(repetition, f32, rows, "repetition", dev),
        0 if frequency is None else vec(frequency, f32, rows, "frequency", dev),
        0 if presence is None else vec(presence, f32, rows, "presence", dev),
        0 if bias_ids is None else vec(bias_ids, i32, None, "bias_ids", dev),
        0 if bias_ids is None else vec(bias, f32, bias_ids.shape[0], "bias", dev),
        0 if bias_ids is None else vec(bias_starts, i64, rows + 1, "bias_starts", dev),
        mp, stride, masks, 0 if row_mask is None else vec(row_mask, i32, rows, "row_mask", dev))
    _serve.check((_serve._lib or _serve.lib()).serve_adjust(
        act, xp, x_row, op, out_row, rows, vocab, lists, _topk._stream(stream)), "serve_adjust")
    return out
