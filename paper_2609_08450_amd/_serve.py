"""Loads libserve_step.so for the modules rotary, evict and logits (include/serve_step.h)."""
from __future__ import annotations

import ctypes
import os
import struct

import torch

from . import paged as _paged
from . import topk as _topk
from .build import SERVE_LIB_PATH

ACTS = {**_paged.ACTS, torch.float32: 2}
PagedError = _paged.PagedError

_P, _i32, _i64, _f32, _size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class Rotary(ctypes.Structure):
    """Mirror of serve_rotary."""

    _fields_ = [("turns", _P), ("magnitude", _f32), ("rot", _i32), ("start", _i32), ("interleaved", _i32)]


class Heads(ctypes.Structure):
    """Mirror of serve_heads."""

    _fields_ = [("in_", _P), ("in_row", _i64), ("in_head", _i64), ("out", _P), ("out_row", _i64), ("out_head", _i64),
                ("heads", _i32)]


class Lists(ctypes.Structure):
    """Mirror of serve_lists."""

    _fields_ = [("tokens", _P), ("token_starts", _P), ("prompt_lens", _P), ("repetition", _P), ("frequency", _P),
                ("presence", _P), ("bias_ids", _P), ("bias", _P), ("bias_starts", _P), ("mask", _P),
                ("mask_stride", _i64), ("n_masks", _i32), ("row_mask", _P)]


# The same as bytes: made in a third of the time of a ctypes structure, and the short calls' host time counts.
pack_heads = struct.Struct("@PqqPqqi4x").pack
pack_lists = struct.Struct("@PPPPPPPPPPqiP").pack

_lib = None


def lib():
    """Loads libserve_step.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(SERVE_LIB_PATH):
            raise PagedError(f"{SERVE_LIB_PATH} is missing: build it with "
                             "`python -m paper_2609_08450_amd.build` (no CPU fallback exists)")
        L = ctypes.CDLL(SERVE_LIB_PATH)
        _topk._check_single_hip_runtime()
        # (structures as addresses: a call hands Heads and Lists over as packed bytes)
        C = R = H = S = _P
        L.serve_rotate.argtypes = [_i32, R, _P, _i32, _i32, _i32, H, H, _i32, _P]
        L.serve_weigh_workspace.argtypes = [_i32, _i32, _i32, _i32]
        L.serve_weigh_workspace.restype = _size
        L.serve_weigh.argtypes = [C, _i32, _P, _i64, _i64, _i32, _P, _P, _i32, _i32, _P, _i32, _P, _i32, _f32, _P, _P,
                                  _P, _size, _P]
        L.serve_keep.argtypes = [_P, _i32, _i32, _P, _i32, _i32, _i32, _P, _i32, _P, _P, _P, _P]
        L.serve_compact.argtypes = [C, _P, _i32, _i32, _P, _i32, _P, _i32, _P]
        L.serve_adjust.argtypes = [_i32, _P, _i64, _P, _i64, _i32, _i32, S, _P]
        for name in ("rotate", "weigh", "keep", "compact", "adjust"):
            getattr(L, "serve_" + name).restype = ctypes.c_int
        _lib = L
    return _lib


STATUS = {-1: "invalid argument", -2: "unsupported size, type or device (gfx950 required)",
          -3: "HIP launch or runtime error", -4: "workspace too small"}


def check(rc: int, what: str):
    if rc != 0:
        raise PagedError(f"{what} failed: {STATUS.get(rc, 'unknown status')} ({rc})")


def empty(shape, like, dtype, stream):
    """An output that a call makes: of the stream that writes it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with _paged._on(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def vec(t, dtype, n, name, dev):
    """Address of a contiguous tensor of one axis, of this type and length (None: any), on device `dev`."""
    if t.dtype is dtype and t.get_device() == dev and t.stride() == (1,) and (n is None or t.shape[0] == n):
        return t.data_ptr()
    return _paged._ptr(t, dtype, (n,), name, dev)


def flat(t, dtype, shape, name, dev):
    """Address of a contiguous tensor of this type and shape (None: any), on device `dev`."""
    if t.dtype is dtype and t.get_device() == dev and (shape is None or t.shape == shape) and t.is_contiguous():
        return t.data_ptr()
    return _paged._ptr(t, dtype, t.shape if shape is None else shape, name, dev)
