"""Plain 64-bit implementations of the calls on either side of the paged cache.
Importing this module does not touch the GPU."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np
import torch

from tests.paged_util import e4m3_round

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half a step of subnormals


def rotated(turns, magnitude, positions, x, start, interleaved, transposed=False):
    """serve_rotate of x [rows, heads, dim] in 64 bits, and |u| + |v| of each element's pair (0 where it is copied).
    `turns`: whole numbers, in units of 2^-64 turns a position; angles are exact until the cosine."""
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    half = len(turns)
    for i, p in enumerate(positions):
        for j, t in enumerate(turns):
            a = (start + 2 * j, start + 2 * j + 1) if interleaved else (start + j, start + half + j)
            angle = 2 * math.pi * float(Fraction((p * t) % 2 ** 64, 2 ** 64))
            c, s = magnitude * math.cos(angle), magnitude * math.sin(angle) * (-1 if transposed else 1)
            u, v = x[i, :, a[0]].double(), x[i, :, a[1]].double()
            y[i, :, a[0]], y[i, :, a[1]] = u * c - v * s, u * s + v * c
            size[i, :, a[0]] = size[i, :, a[1]] = u.abs() + v.abs()
    return y, size


def assert_rotated(got, ref, magnitude, where=""):
    """The cosine is off by at most 2^-22 (two units in the last place of 1, the angle's 2^-25 of an eighth of a
    turn), its product with the magnitude, those of the pair and their sum by 2^-24 of their size each; the
    result by half a step of its type.  Copied elements are the same."""
    y, size = ref
    got = got.cpu()
    tol = 2.0 ** -21 * magnitude * size
    tol += torch.where(size > 0, HALF_STEP[got.dtype] * (y.abs() + tol) + LEAST[got.dtype], 0.0)
    off = (got.double() - y).abs()
    assert bool((off <= tol).all()), f"{where}: {float((off - tol).max()):.3g} out of bounds"


def weighed(s, lse, scale=None):
    """What serve_weigh adds for a paged_util.Setup: for each request, its tokens' sums in 64 bits, the bound of
    their error, and which tokens are in the cache.

    The bound, for each p = exp(x - lse): products of q and k are exact, their FP32 sum of D terms is off by at
    most D 2^-24 of the sum of magnitudes; the factors scale * log2(e) * page scale and lse * log2(e), three and
    two roundings, by 2^-22 of x and of lse; the exponent's sum by 2^-24 of itself, exp2 by two units: p is off by
    p times that.  A sum of N of them by N 2^-24 of itself."""
    scale = s.scale if scale is None else scale
    cap = s.table.shape[1] * s.page
    G = s.heads // s.kv
    starts = s.row_starts.tolist()
    sums, bounds, held = [], [], []
    for r in range(len(starts) - 1):
        rows = range(min(max(starts[r], 0), s.n_rows), min(max(starts[r + 1], 0), s.n_rows))
        lens = [min(max(int(s.row_lengths[i]), 0), cap) for i in rows]
        L = max([0, *lens])
        total = torch.zeros(L, dtype=torch.float64, device=s.q.device)
        bound, there = total.clone(), torch.ones(L, dtype=torch.bool, device=s.q.device)
        if L:
            k, there = s.tokens("k", r, L)
            k = torch.where(there[:, None], k, 0.0)
            for i, n in zip(rows, lens):
                for h in range(s.heads):
                    z = float(lse[i, h])
                    if n == 0 or z == -math.inf:
                        continue
                    q = s.q[i, h].double()
                    x = scale * torch.matmul(k[h // G, :n], q)
                    size = scale * torch.matmul(k[h // G, :n].abs(), q.abs())
                    p = torch.exp(x - z)
                    total[:n] += p
                    bound[:n] += p * (s.dim * 2.0 ** -24 * size + 2.0 ** -22 * (x.abs() + abs(z)) + 2.0 ** -21)
            bound += total * len(rows) * s.heads * 2.0 ** -24
        sums.append(total)
        bounds.append(bound)
        held.append(there)
    return sums, bounds, held


def kept(idx, lens, first, last, base):
    """Ascending numbers of the tokens that stay, of each request."""
    out = []
    for row, L in zip(idx, lens):
        stay = {base + i for i in row if i >= 0} | set(range(first)) | set(range(max(L - last, 0), max(L, 0)))
        out.append(sorted(i for i in stay if i < L))
    return out


def compacted(codes, scale, table, lists, page, dtype):
    """serve_compact of one side: codes as numbers float64 [pages, heads, page, dim], scale float32 [pages, heads]."""
    f32 = np.float32
    old_codes, old_scale = codes.copy(), scale.copy()
    codes, scale = codes.copy(), scale.copy()
    n_pages = len(codes)
    for r, tokens in enumerate(lists):
        tokens = tokens[:len(table[r]) * page]
        for p in range(-(-len(tokens) // page)):
            part = tokens[p * page:(p + 1) * page]
            to = table[r][p]
            if part[-1] == p * page + len(part) - 1 or not 0 <= to < n_pages:
                continue
            for h in range(codes.shape[1]):
                x, s = np.zeros((len(part), codes.shape[3])), np.zeros((len(part), 1), f32)
                for i, t in enumerate(part):
                    at = table[r][t // page]
                    if 0 <= at < n_pages:
                        x[i], s[i] = old_codes[at, h, t % page], old_scale[at, h]
                top = f32((np.abs(x).astype(f32) * s).max())
                if dtype is torch.int8:
                    new = max(top * (f32(1) / f32(127)), f32(2.0 ** -100))
                    # exact products, one rounding of the quotient in 64 bits: a tie stays one
                    y = np.clip(np.rint(x * s.astype(np.float64) / np.float64(new)), -127, 127)
                else:
                    new = f32(2.0 ** -100)
                    while f32(448) * new < top:
                        new *= f32(2)
                    y = e4m3_round(((x.astype(f32) * s) / new).astype(np.float64))
                codes[to, h, :len(part)] = y
                scale[to, h] = new
    return codes, scale


def adjusted(x, tokens=None, prompt=0, repetition=1.0, frequency=0.0, presence=0.0, biases=None, allowed=None):
    """serve_adjust of one row: x float32 [vocab]; biases a list of (id, value); allowed truth values."""
    f32 = np.float32
    x = x.astype(f32).copy()
    vocab = len(x)
    with np.errstate(all="ignore"):
        for t in set(tokens or []):
            if 0 <= t < vocab:
                x[t] = x[t] / f32(repetition) if x[t] > 0 else x[t] * f32(repetition)
        said = list(tokens or [])[max(prompt, 0):]
        for t in set(said):
            if 0 <= t < vocab:
                x[t] = (x[t] - f32(frequency) * f32(said.count(t))) - f32(presence)
        for t, b in dict(biases or []).items():
            if 0 <= t < vocab:
                x[t] = x[t] + f32(b)
    if allowed is not None:
        x[~allowed] = -np.inf
    return x


def mask_words(allowed):
    """Truth values [masks, vocab] as int32 words of bits."""
    n, vocab = allowed.shape
    words = -(-vocab // 32)
    padded = np.zeros((n, words * 32), np.uint8)
    padded[:, :vocab] = allowed
    bits = np.packbits(padded.reshape(n, words, 32), axis=-1, bitorder="little")
    return bits.view("<u4").reshape(n, words).view(np.int32)
