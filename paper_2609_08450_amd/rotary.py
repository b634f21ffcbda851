"""Rotary positions for queries and keys, before ``paged.store``, ``paged.attend`` and ``paged.score``.

A ``Rotary`` holds the frequencies that a model keeps; ``rotate`` forwards to
serve_rotate() (include/serve_step.h), which has the contract.  As in ``paged``,
all work runs in the library's HIP kernels, on ``stream`` or the current one, and
errors are ``paged.PagedError``::

    rope = rotary.Rotary(128, base=1e6, scaling="yarn", factor=4.0, original=32768)
    rotary.rotate(rope, positions, q, k, q_out=q, k_out=k)     # in place
    paged.store(cache, k, v, slots)
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _serve
from . import paged as _paged
from . import topk as _topk

PagedError = _paged.PagedError
LAYOUTS = {"half": 0, "interleaved": 1}


def frequencies(rot: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                original: int | None = None, *, fast: float = 32.0, slow: float = 1.0, low: float = 1.0,
                high: float = 4.0) -> tuple[list[float], float]:
    """Radians a position of each of the rot / 2 pairs, and the magnitude that goes with them.

    None       f_p = base^(-2 p / rot)
    "linear"   f_p / factor: positions are interpolated
    "ntk"      base * factor^(rot / (rot - 2)) in base's place: the slowest pair is scaled by the
               whole factor, the fastest not at all
    "yarn"     pairs that turn more than `fast` times over the original context keep f_p, those
               that turn less than `slow` times get f_p / factor, with a ramp over the pairs between;
               magnitude 0.1 ln(factor) + 1 (for factors above 1)
    "bands"    t = turns over the original context: f_p where t >= high, f_p / factor where
               t <= low, between them mixed in proportion to t
    """
    if rot < 2 or rot % 2:
        raise PagedError(f"rot must be even and at least 2, got {rot}")
    if not (base > 0 and math.isfinite(base)):
        raise PagedError(f"base must be positive, got {base}")
    if scaling not in (None, "linear", "ntk", "yarn", "bands"):
        raise PagedError(f"scaling must be None, 'linear', 'ntk', 'yarn' or 'bands', got {scaling!r}")
    if scaling is not None and not (factor > 0 and math.isfinite(factor)):
        raise PagedError(f"factor must be positive, got {factor}")
    if scaling in ("yarn", "bands") and not (original and original > 0):
        raise PagedError(f"{scaling!r} needs the original context length")
    if scaling == "ntk":
        if rot == 2:
            raise PagedError("'ntk' needs more than one pair")
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2 * p / rot) for p in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "yarn":
        if base == 1.0 or not fast > slow > 0:
            raise PagedError("'yarn' needs a base other than 1, and fast > slow > 0")

        def pair(turns):
            """The (fractional) pair that turns so often over the original context."""
            return rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))

        first, last = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot - 1)
        ramp = [min(max((p - first) / max(last - first, 0.001), 0.0), 1.0) for p in range(rot // 2)]
        return [x / factor * m + x * (1 - m) for x, m in zip(f, ramp)], 0.1 * math.log(factor) + 1 if factor > 1 else 1.0
    if scaling == "bands":
        if not high > low > 0:
            raise PagedError("'bands' needs high > low > 0")
        keep = [min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        return [x / factor * (1 - m) + x * m for x, m in zip(f, keep)], 1.0
    return f, 1.0


class Rotary:
    """The frequencies of one kind of head: `rot` elements from `start` on are rotated, in pairs of
    elements p and p + rot / 2 (``layout="half"``) or 2 p and 2 p + 1 (``"interleaved"``).
    The arguments of ``frequencies`` follow; ``magnitude`` overrides its own."""

    def __init__(self, rot: int, *, base: float = 10000.0, layout: str = "half", start: int = 0,
                 scaling: str | None = None, factor: float = 1.0, original: int | None = None,
                 magnitude: float | None = None, device="cuda", **bounds):
        f, m = frequencies(rot, base, scaling, factor, original, **bounds)
        self._set(f, m if magnitude is None else magnitude, layout, start, device)

    @classmethod
    def of(cls, frequencies, magnitude: float = 1.0, layout: str = "half", start: int = 0, device="cuda") -> "Rotary":
        """Of a program's own frequencies, in radians a position (floats of any size)."""
        self = cls.__new__(cls)
        self._set([float(x) for x in frequencies], magnitude, layout, start, device)
        return self

    def _set(self, f, magnitude, layout, start, device):
        if layout not in LAYOUTS:
            raise PagedError(f"layout must be 'half' or 'interleaved', got {layout!r}")
        if start < 0 or not 1 <= len(f) <= 512:
            raise PagedError("start must not be negative, and from 2 to 1024 elements are rotated")
        if not all(map(math.isfinite, f)) or not math.isfinite(magnitude):
            raise PagedError("frequencies and the magnitude must be finite")
        self.frequencies, self.magnitude, self.layout, self.start = f, float(magnitude), layout, start
        self.rot = 2 * len(f)
        # turns a position, in units of 2^-64, as the signed numbers with the same bits
        turns = [int(math.fmod(x / (2 * math.pi), 1.0) * 2.0 ** 64) % 2 ** 64 for x in f]
        self.turns = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64, device=device)
        self._device = self.turns.get_device()
        self._c = _serve.Rotary(self.turns.data_ptr(), self.magnitude, self.rot, start, LAYOUTS[layout])
        self._at = ctypes.addressof(self._c)


def _check_heads(x, name, dtype, shape, dev):
    """What makes heads [rows, heads, dim] unfit."""
    if x.get_device() != dev:
        raise _paged._elsewhere(x, dev, name)
    if x.dtype is not dtype or tuple(x.shape) != shape:
        raise PagedError(f"{name} must be {dtype} of shape {shape}, got {x.dtype} {tuple(x.shape)}")
    if x.numel() and shape[2] > 1 and x.stride(2) != 1:
        raise PagedError(f"{name} must have a contiguous last axis")


def _heads(x, out, name, dtype, rows, dim, dev, stream):
    """The output, and serve_heads as bytes."""
    shape, at = x.shape, x.stride()
    if x.get_device() != dev or x.dtype is not dtype or len(shape) != 3 or shape[0] != rows or shape[2] != dim or at[2] != 1:
        _check_heads(x, name, dtype, (rows, shape[1] if len(shape) == 3 else "heads", dim), dev)
    heads = shape[1]
    if out is x:
        to = at
    elif out is None:
        out = _serve.empty(shape, x, dtype, stream)
        to = (heads * dim, dim, 1)
    else:
        to = out.stride()
        if out.get_device() != dev or out.dtype is not dtype or out.shape != shape or to[2] != 1:
            _check_heads(out, name + "_out", dtype, tuple(shape), dev)
    if 0 in to and any(n > 1 and s == 0 for n, s in zip(shape, to)) and x.numel():
        raise PagedError(f"{name}_out must not be an expanded tensor")
    row, head, to_row, to_head = at[0], at[1], to[0], to[1]
    if rows == 1:  # the stride of an axis of length one says nothing
        row = to_row = 0
    if heads == 1:
        head = to_head = 0
    return out, _serve.pack_heads(x.data_ptr(), row, head, out.data_ptr(), to_row, to_head, heads)


def rotate(rotary: Rotary, positions, q, k=None, *, q_out=None, k_out=None, transposed: bool = False, stream=None):
    """Forwards to serve_rotate(): q [rows, heads, dim] (and k, of the same type and rows) at ``positions``
    (int32 or int64 [rows]), bfloat16, float16 or float32.  ``q_out`` and ``k_out`` may be q and k
    themselves; where they are not given they are made.  ``transposed`` turns the other way: the gradient's
    direction.  Returns q_out, or (q_out, k_out) with a k."""
    dev = _paged._device(q, "q")
    if rotary._device != dev:
        raise PagedError(f"the rotary frequencies are on cuda:{rotary._device}, q is on cuda:{dev}")
    dtype, shape = q.dtype, q.shape
    act = _serve.ACTS.get(dtype)
    if act is None or len(shape) != 3:
        raise PagedError(f"q must be bfloat16, float16 or float32 [rows, heads, dim], got {dtype} {tuple(shape)}")
    rows, _, dim = shape
    wide = positions.dtype is torch.int64
    at = _serve.vec(positions, torch.int64 if wide else torch.int32, rows, "positions", dev)
    q_out, qh = _heads(q, q_out, "q", dtype, rows, dim, dev, stream)
    kh = None
    if k is not None:
        k_out, kh = _heads(k, k_out, "k", dtype, rows, dim, dev, stream)
    elif k_out is not None:
        raise PagedError("k_out belongs to a k")
    _serve.check((_serve._lib or _serve.lib()).serve_rotate(
        act, rotary._at, at, wide, rows, dim, qh, kh, transposed, _topk._stream(stream)), "serve_rotate")
    return q_out if k is None else (q_out, k_out)
