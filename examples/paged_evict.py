"""Serving steps with a cache of bounded length on one GPU: every call as a program makes it.

    python examples/paged_evict.py [--requests N] [--context L] [--budget B] [--steps S]

One layer of a model with random weights: for each step
tables -> rotate -> store -> attend -> weigh, then logits -> adjust -> Top-K -> a token drawn.
When a request may have passed the budget, the tokens with the largest weights stay
beside its first and its last ones: Top-K -> keep -> compact -> tables, which takes the
free pages back.  Positions go on counting: a token keeps the one that it was stored with.
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

from examples.paged_step import Server  # noqa: E402
from paper_2609_08450_amd import evict, logits, paged, rotary, topk  # noqa: E402


class Layer:
    """One layer's cache, and the weight that each of its tokens has had."""

    def __init__(self, server, page=64, heads=16, kv_heads=2, dim=128):
        requests, self.max_len = server.table.shape[0], server.width * page
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.cache = paged.PagedCache(server.n_pages, page, kv_heads, dim)
        self.weights = torch.zeros((requests, self.max_len), device="cuda")
        self.offsets = torch.arange(requests, device="cuda") * self.max_len


class Eviction:
    """Brings requests down to `budget` tokens: the first, the last, and by weight between them."""

    def __init__(self, requests, budget, first=4, last=64):
        self.first, self.last, self.budget = first, last, budget
        self.select = topk.TopK(requests, budget - first - last)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.kept, self.counts = torch.empty((requests, budget), **i32), torch.empty(requests, **i32)

    def __call__(self, server, layer):
        between = (server.lens - self.first - self.last).clamp(min=0)
        idx, _ = self.select(layer.weights, layer.offsets + self.first, between)
        evict.keep(idx, server.lens, self.first, self.last, self.kept, self.counts, base=self.first,
                   weights=layer.weights, weight_offsets=layer.offsets)
        evict.compact(layer.cache, server.table, self.kept, self.counts)
        server.begin(self.counts - server.lens, 0)


class Sampler:
    """Draws each request's next token, with penalties on those that it has."""

    def __init__(self, requests, max_tokens, vocab, K=64, repetition=1.1, presence=0.2):
        self.tokens = torch.full((requests, max_tokens), -1, dtype=torch.int32, device="cuda")  # -1: none yet
        self.starts = torch.arange(requests + 1, device="cuda") * max_tokens
        self.repetition = torch.full((requests,), repetition, device="cuda")
        self.presence = torch.full((requests,), presence, device="cuda")
        self.offsets = torch.arange(requests, device="cuda") * vocab
        self.lengths = torch.full((requests,), vocab, dtype=torch.int32, device="cuda")
        self.select = topk.TopK(requests, K)

    def __call__(self, x, prompt_lens, generator=None):
        rows = logits.adjust(x, tokens=self.tokens.view(-1), token_starts=self.starts, prompt_lens=prompt_lens,
                             repetition=self.repetition, presence=self.presence)
        idx, val = self.select(rows, self.offsets, self.lengths)
        drawn = torch.multinomial(torch.softmax(val, -1), 1, generator=generator)
        return idx.gather(1, drawn).view(-1)


def attention(server, layer, rope, positions, q, k, v):
    """One layer's attention of a step, with its tokens' weights."""
    rotary.rotate(rope, positions, q, k, q_out=q, k_out=k)
    paged.store(layer.cache, k, v, server.slots)
    lse = torch.empty(q.shape[:2], device="cuda")
    scale = layer.dim ** -0.5
    out = paged.attend(layer.cache, q, server.table, server.row_starts, server.row_lengths, scale, lse=lse)
    evict.weigh(layer.cache, q, lse, server.table, server.row_starts, server.row_lengths, scale, layer.weights,
                layer.offsets)
    return out


class Model:
    """An embedding, one layer's projections and the answer's, all random."""

    def __init__(self, heads, kv_heads, dim, vocab=32000, width=512, max_position=1 << 17, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def r(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * shape[-2] ** -0.5).to(torch.bfloat16)

        self.heads, self.kv_heads, self.dim, self.vocab = heads, kv_heads, dim, vocab
        self.embedding = torch.randn((vocab, width), generator=g, device="cuda").to(torch.bfloat16)
        self.qkv = r(width, (heads + 2 * kv_heads) * dim)
        self.answer = r(heads * dim, vocab)
        self.rope = rotary.Rotary(dim, base=1e6, scaling="yarn", factor=4.0, original=max_position // 4)

    def projected(self, tokens):
        x = (self.embedding[tokens.long()] @ self.qkv).view(tokens.numel(), -1, self.dim)
        return x.split([self.heads, self.kv_heads, self.kv_heads], 1)


def run(requests=8, context=8192, budget=2048, steps=64, chunk=4096, slack=64, vocab=32000, seed=0):
    """Prompts of about `context` tokens, each brought down to `budget`, then `steps` tokens of each request,
    brought down again every `slack` steps.  Returns the server, the layer, the tokens and the seconds a step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    server = Server(requests, context + slack + 64)
    layer = Layer(server)
    model = Model(layer.heads, layer.kv_heads, layer.dim, vocab)
    evicted = Eviction(requests, budget)
    sampler = Sampler(requests, context + steps + 1, vocab)
    positions = torch.zeros(requests, dtype=torch.int32, device="cuda")
    last = torch.zeros((requests, layer.heads * layer.dim), dtype=torch.bfloat16, device="cuda")
    new = torch.zeros(requests, dtype=torch.int32, device="cuda")
    prompts = [max(1, context - 7 * r) for r in range(requests)]
    for r, length in enumerate(prompts):
        sampler.tokens[r, :length] = torch.randint(vocab, (length,), generator=g, device="cuda", dtype=torch.int32)
        for at in range(0, length, chunk):
            rows = min(chunk, length - at)
            new.zero_()
            new[r] = rows
            server.begin(new, rows)
            q, k, v = model.projected(sampler.tokens[r, at:at + rows])
            out = attention(server, layer, model.rope, torch.arange(at, at + rows, device="cuda"), q, k, v)
        last[r] = out[-1].flatten()
        positions[r] = length
    evicted(server, layer)
    new.fill_(1)
    prompt_lens = positions.clone()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for step in range(steps):
        token = sampler(last @ model.answer, prompt_lens, g)
        sampler.tokens.scatter_(1, positions.long()[:, None], token[:, None])
        server.begin(new, requests)
        q, k, v = model.projected(token)
        last = attention(server, layer, model.rope, positions, q, k, v).flatten(1)
        positions += 1
        if (step + 1) % slack == 0:
            evicted(server, layer)
    torch.cuda.synchronize()
    return server, layer, sampler.tokens, (time.perf_counter() - began) / max(1, steps)


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--requests", type=int, default=8)
    p.add_argument("--context", type=int, default=8192)
    p.add_argument("--budget", type=int, default=2048)
    p.add_argument("--steps", type=int, default=64)
    a = p.parse_args()
    server, layer, tokens, spent = run(a.requests, a.context, a.budget, a.steps)
    print(f"{a.requests} requests, {a.context} tokens each, {int(server.lens.max())} of them kept in "
          f"{server.n_pages - int(server.pool[1])} pages: {spent * 1e6:.1f} us a step of one layer")
