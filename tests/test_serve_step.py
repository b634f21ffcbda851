"""The serving step's calls together, as the example makes them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def values(cache, scale, codes, table, request, length, page):
    """A request's tokens [heads, length, dim] of one side of the cache, in 64 bits."""
    pages = table[request, :-(-length // page)].long()
    x = codes.view(torch.uint8)[pages].view(codes.dtype).float().double() * scale[pages].double()[..., None, None]
    return x.transpose(0, 1).flatten(1, 2)[:, :length]


def test_weights_evict_and_the_tables_take_the_pages():
    """Prompts of 900 and 100 tokens, a budget of 300: rows of attention sum to one, the selection's tokens stay
    with their weights and values, and pages go back to the ring."""
    from examples import paged_evict

    server = paged_evict.Server(2, 1024)
    layer = paged_evict.Layer(server)
    model = paged_evict.Model(layer.heads, layer.kv_heads, layer.dim, vocab=500, width=64)
    evicted = paged_evict.Eviction(2, 300, first=4, last=50)
    g = torch.Generator(device="cuda").manual_seed(1)
    lens = [900, 100]
    server.begin(torch.tensor(lens, dtype=torch.int32, device="cuda"), 1000)
    q, k, v = model.projected(torch.randint(500, (1000,), generator=g, device="cuda"))
    positions = torch.cat([torch.arange(n, device="cuda") for n in lens])
    paged_evict.attention(server, layer, model.rope, positions, q, k, v)
    # Each row and head hands out 1, but for what attend's lse is off by (2^-15 (1 + |lse|), |lse| < 8) and the
    # exponents here: FP32 sums of 128 products, at most 128 2^-24 of their magnitudes' sum, about 8; 2^-12 and
    # 2^-14 with the roundings of the sums.
    for r, n in enumerate(lens):
        assert abs(float(layer.weights[r].double().sum()) / (n * layer.heads) - 1) <= 2.0 ** -11
        assert bool((layer.weights[r, n:] == 0).all()) and bool((layer.weights[r, :n] > 0).all())
    before, table = layer.weights.cpu(), server.table.clone()
    sides = [(layer.cache.k, layer.cache.k_scale), (layer.cache.v, layer.cache.v_scale)]
    old = [[values(layer.cache, s, c, table, r, n, 64) for c, s in sides] for r, n in enumerate(lens)]
    evicted(server, layer)
    assert server.lens.tolist() == [300, 100]
    assert server.n_pages - int(server.pool[1]) == 5 + 2  # pages of 64
    for r, n in enumerate(lens):
        m = min(n, 300)
        kept = evicted.kept[r, :m].cpu().long()
        if n > 300:
            best = torch.topk(before[r, 4:n - 50], 300 - 54).indices + 4
            want = torch.cat([torch.arange(4), best, torch.arange(n - 50, n)]).sort().values
            assert torch.equal(before[r, kept].sort().values, before[r, want].sort().values)
        else:
            assert torch.equal(kept, torch.arange(n))
        assert torch.equal(layer.weights[r, :m].cpu(), before[r, kept])
        assert bool((layer.weights[r, m:n] == 0).all())
        for (codes, scale), was in zip(sides, old[r]):
            x, want = values(layer.cache, scale, codes, server.table, r, m, 64), was[:, kept.cuda()]
            # e4m3's scales are powers of two, at most 2 / 448 of a page's largest value: only steps of the least
            # size, 2^-9 of a scale, round, by half of one
            assert bool(((x - want).abs() <= 2.0 ** -10 * 2 / 448 * was.abs().amax()).all())


def test_the_example_runs_on_after_eviction():
    from examples import paged_evict

    server, layer, tokens, _ = paged_evict.run(requests=3, context=700, budget=256, steps=20, chunk=300, slack=8, vocab=1000)
    # 20 steps: down to 256 at the 16th, four more after it
    assert server.lens.tolist() == [260] * 3
    assert server.n_pages - int(server.pool[1]) == 3 * 5
    made = [tokens[r, 700 - 7 * r:720 - 7 * r] for r in range(3)]
    assert all(bool(((t >= 0) & (t < 1000)).all()) for t in made) and int(tokens[0, 720]) == -1
    assert torch.isfinite(layer.weights).all() and bool((layer.weights[:, 260:] == 0).all())


def test_a_captured_step_is_the_eager_one():
    """Two steps, an eviction and a choice of tokens in one graph, against the same calls without one: five times,
    with work of other kinds between them, from the same state, to the bit."""
    from examples import paged_evict

    class State:
        def __init__(self):
            self.server = paged_evict.Server(4, 640)
            self.layer = paged_evict.Layer(self.server)
            self.model = paged_evict.Model(self.layer.heads, self.layer.kv_heads, self.layer.dim, vocab=700, width=64)
            self.evicted = paged_evict.Eviction(4, 200, first=2, last=30)
            self.sampler = paged_evict.Sampler(4, 40, 700, K=8)
            self.positions = torch.tensor([220, 90, 300, 201], dtype=torch.int32, device="cuda")
            self.new = torch.ones(4, dtype=torch.int32, device="cuda")
            self.prompt = torch.zeros(4, dtype=torch.int32, device="cuda")
            self.token = torch.zeros(4, dtype=torch.int32, device="cuda")
            g = torch.Generator(device="cuda").manual_seed(2)
            rows = int(self.positions.sum())
            self.server.begin(self.positions, rows)
            positions = torch.cat([torch.arange(n, device="cuda") for n in self.positions.tolist()])
            x = self.model.projected(torch.randint(700, (rows,), generator=g, device="cuda"))
            paged_evict.attention(self.server, self.layer, self.model.rope, positions, *x)

        def steps(self):
            for _ in range(2):
                self.server.begin(self.new, 4)
                x = self.model.projected(self.token)
                out = paged_evict.attention(self.server, self.layer, self.model.rope, self.positions, *x)
                self.positions += 1
                rows = paged_evict.logits.adjust(
                    out.flatten(1) @ self.model.answer, tokens=self.sampler.tokens.view(-1),
                    token_starts=self.sampler.starts, prompt_lens=self.prompt, repetition=self.sampler.repetition,
                    presence=self.sampler.presence)
                idx, _ = self.sampler.select(rows, self.sampler.offsets, self.sampler.lengths)
                # the likeliest joins the tokens so far, of equal ones the first (the selection has them in any order)
                score = rows.gather(1, idx.long())
                self.token.copy_(torch.where(score == score.amax(1, keepdim=True), idx, 700).amin(1))
                self.sampler.tokens.scatter_(1, self.positions.long()[:, None] % 40, self.token[:, None])
            self.evicted(self.server, self.layer)
            # (an odd number of tables in all: the lengths go back to where the next call looks)
            self.server.lens, self.server.next_lens = self.server.next_lens.copy_(self.server.lens), self.server.lens

        def seen(self):
            s, c = self.server, self.layer.cache
            return [t.clone() for t in (s.lens, s.pool, s.ring, s.table, self.layer.weights, c.k.view(torch.uint8),
                                        c.v.view(torch.uint8), c.k_scale, c.v_scale, self.token, self.sampler.tokens)]

    eager, captured = State(), State()
    eager.steps()
    captured.steps()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.steps()
    for i in range(5):
        graph.replay()
        eager.steps()
        torch.rand((300, 300), device="cuda").sum()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.seen(), captured.seen())), i
    assert eager.server.lens.tolist() == [200, 102, 200, 200]
