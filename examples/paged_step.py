"""Serving steps of sparse attention on one GPU: every call of the chain as a program makes it.

    python examples/paged_step.py [--requests N] [--context L] [--steps S]

One layer of a model with random weights' activations: a paged 8-bit cache of
keys and values, an indexer's cache of keys alone, and for each step
tables -> store (both caches) -> score -> Top-K -> attention over the selected
tokens.  The first step is the prompts, in chunks; then come single tokens.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2609_08450_amd import paged, topk  # noqa: E402


class Layer:
    """One layer's caches and the sizes of its heads."""

    def __init__(self, n_pages, page=64, heads=16, kv_heads=2, dim=128, index_heads=8, index_dim=64, K=2048):
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.index_heads, self.index_dim, self.K = index_heads, index_dim, K
        self.cache = paged.PagedCache(n_pages, page, kv_heads, dim)
        self.index = paged.PagedCache(n_pages, page, 1, index_dim, values=False)


class Server:
    """Pages, lengths and block tables of up to `requests` requests, shared by all layers."""

    def __init__(self, requests, max_len, page=64, n_pages=None):
        self.page, self.width = page, -(-max_len // page)
        n_pages = n_pages or requests * self.width
        i32 = dict(dtype=torch.int32, device="cuda")
        self.n_pages = n_pages
        self.ring = torch.arange(n_pages, **i32)
        self.pool = torch.tensor([0, n_pages, 0, 0], **i32)
        self.table = torch.full((requests, self.width), -1, **i32)
        self.lens, self.next_lens = torch.zeros(requests, **i32), torch.zeros(requests, **i32)
        self.row_starts = torch.empty(requests + 1, **i32)

    def begin(self, new_lens, rows):
        """A step's tables: new_lens int32 [requests] on the GPU, `rows` their sum."""
        self.row_request, self.row_lengths = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        self.slots = torch.empty(rows, dtype=torch.int64, device="cuda")
        paged.tables(self.ring, self.pool, self.lens, new_lens, self.table, self.page, pool_out=self.pool,
                     lens_out=self.next_lens, row_starts=self.row_starts, row_request=self.row_request,
                     row_lengths=self.row_lengths, slots=self.slots)
        self.lens, self.next_lens = self.next_lens, self.lens


class Selector:
    """Score rows and a selection for up to `max_rows` rows."""

    def __init__(self, max_rows, max_len, K):
        self.pitch = -(-max_len // 32) * 32
        self.scores = torch.empty((max_rows, self.pitch), device="cuda")
        self.offsets = torch.arange(max_rows, device="cuda") * self.pitch
        self.topk = topk.TopK(max_rows, K)


def sparse_attention(server, layer, selector, k, v, q, index_k, index_q, index_w):
    """One layer's attention of a step: stores, scores, selects, attends."""
    rows = q.shape[0]
    paged.store(layer.cache, k, v, server.slots)
    paged.store(layer.index, index_k, None, server.slots)
    offsets = selector.offsets[:rows]
    paged.score(layer.index, index_q, index_w, server.table, server.row_request, server.row_lengths,
                layer.index_dim ** -0.5, selector.scores, offsets)
    idx, _ = selector.topk(selector.scores, offsets, server.row_lengths)
    return paged.attend_selected(layer.cache, q, idx, server.table, server.row_request, server.row_lengths,
                                 layer.dim ** -0.5)


def dense_attention(server, layer, q):
    """The same rows over everything that their requests hold."""
    return paged.attend(layer.cache, q, server.table, server.row_starts, server.row_lengths, layer.dim ** -0.5)


def activations(layer, rows, g):
    """Keys and values, queries, and the indexer's of `rows` tokens."""
    def r(*shape):
        return torch.randn((rows, *shape), generator=g, device="cuda").to(torch.bfloat16)

    return dict(k=r(layer.kv_heads, layer.dim), v=r(layer.kv_heads, layer.dim), q=r(layer.heads, layer.dim),
                index_k=r(1, layer.index_dim), index_q=r(layer.index_heads, layer.index_dim),
                index_w=torch.rand((rows, layer.index_heads), generator=g, device="cuda"))


def run(requests=8, context=8192, steps=16, K=2048, chunk=4096, seed=0):
    """Prompts of about `context` tokens, then `steps` single tokens of each request.
    Returns the last step's sparse and dense outputs and its seconds a step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    max_len = context + steps
    server = Server(requests, max_len)
    layer = Layer(server.n_pages, K=K)
    selector = Selector(max(requests, chunk), max_len, K)
    new = torch.zeros(requests, dtype=torch.int32, device="cuda")
    for r in range(requests):
        left = context - 7 * r
        while left > 0:
            rows = min(chunk, left)
            new.zero_()
            new[r] = rows
            server.begin(new, rows)
            sparse_attention(server, layer, selector, **activations(layer, rows, g))
            left -= rows
    new.fill_(1)
    acts = [activations(layer, requests, g) for _ in range(steps)]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for x in acts:
        server.begin(new, requests)
        sparse = sparse_attention(server, layer, selector, **x)
    torch.cuda.synchronize()
    spent = (time.perf_counter() - began) / max(1, steps)
    return sparse, dense_attention(server, layer, acts[-1]["q"]), spent


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--requests", type=int, default=8)
    p.add_argument("--context", type=int, default=8192)
    p.add_argument("--steps", type=int, default=16)
    a = p.parse_args()
    sparse, dense, spent = run(a.requests, a.context, a.steps)
    print(f"{a.requests} requests, {a.context} tokens each: {spent * 1e6:.1f} us a step of one layer; "
          f"sparse and dense outputs differ by {float((sparse.float() - dense.float()).norm() / dense.float().norm()):.3f} of their norm")
