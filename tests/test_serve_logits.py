"""Penalties, biases and masks on logits against their definition: equal to the bit, since every step of it is
rounded to FP32."""
import numpy as np
import pytest
import torch

from tests.serve_util import adjusted, mask_words

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def ragged(lists, dtype):
    starts = np.cumsum([0, *map(len, lists)])
    return (torch.tensor([x for row in lists for x in row], dtype=dtype).cuda(), torch.tensor(starts, dtype=torch.int64).cuda())


class Case:
    """Seeded rows: tokens of a small part of the vocabulary, so that they repeat, ids outside it among them."""

    def __init__(self, rows, vocab, act=torch.float32, history=50, biases=20, masks=3, pitch=None, out_pitch=None, seed=0,
                 special=False):
        g = np.random.default_rng(seed)
        self.rows, self.vocab = rows, vocab
        wide = torch.from_numpy(4 * g.standard_normal((rows, pitch or vocab)).astype(np.float32)).to(act).cuda()
        self.x = wide[:, :vocab]
        if special:
            at = g.integers(0, vocab, (rows, 40))
            for r in range(rows):
                self.x[r, at[r, :10]], self.x[r, at[r, 10:20]] = np.inf, -np.inf
                self.x[r, at[r, 20:30]], self.x[r, at[r, 30:]] = 0.0, -0.0
        self.wide, self.out_wide = wide, torch.full((rows, out_pitch or vocab), 9.0, device="cuda")
        self.out = self.out_wide[:, :vocab]
        self.how = {}
        few = max(1, vocab // 3)
        self.tokens = [g.integers(-2, few, g.integers(0, history + 1)).tolist() + ([vocab, vocab - 1, 2 ** 31 - 1, -2 ** 31]
                       if history else []) for _ in range(rows)]
        self.prompts = [int(g.integers(0, len(t) + 2)) for t in self.tokens]
        self.rep, self.freq, self.pres = (g.uniform(a, b, rows).astype(np.float32) for a, b in ((0.5, 2), (-1, 1), (-1, 1)))
        if history:
            self.how["tokens"], self.how["token_starts"] = ragged(self.tokens, torch.int32)
            self.how.update(prompt_lens=torch.tensor(self.prompts, dtype=torch.int32).cuda(),
                            repetition=torch.from_numpy(self.rep).cuda(), frequency=torch.from_numpy(self.freq).cuda(),
                            presence=torch.from_numpy(self.pres).cuda())
        counts = [int(n) for n in g.integers(0, biases + 1, rows)]
        self.biases = [list(zip(g.integers(-1, vocab + 1, n).tolist(),
                                (3 * g.standard_normal(n)).astype(np.float32).tolist())) for n in counts]
        if biases:
            self.how["bias_ids"], self.how["bias_starts"] = ragged([[i for i, _ in b] for b in self.biases], torch.int32)
            self.how["bias"] = ragged([[v for _, v in b] for b in self.biases], torch.float32)[0]
        self.allowed = g.random((masks, vocab)) < 0.4 if masks else None
        self.row_mask = g.integers(-2, masks + 2, rows).tolist() if masks else None
        if masks:
            self.how["mask"] = torch.from_numpy(mask_words(self.allowed)).cuda()
            self.how["row_mask"] = torch.tensor(self.row_mask, dtype=torch.int32).cuda()

    def ref(self, x=None):
        x = (self.x if x is None else x).float().cpu().numpy()
        out = np.empty_like(x)
        for r in range(self.rows):
            m = self.row_mask[r] if self.row_mask else -1
            out[r] = adjusted(x[r], self.tokens[r] if "tokens" in self.how else None, self.prompts[r], self.rep[r],
                              self.freq[r], self.pres[r], self.biases[r],
                              self.allowed[m] if self.allowed is not None and 0 <= m < len(self.allowed) else None)
        return out

    def check(self, **change):
        from paper_2609_08450_amd import logits

        ref = self.ref()
        around = self.out_wide.clone()
        got = logits.adjust(self.x, self.out, **{**self.how, **change})
        assert got is self.out
        torch.cuda.synchronize()
        assert same(got, ref)
        assert torch.equal(self.out_wide[:, self.vocab:], around[:, self.vocab:])


def same(got, ref):
    """Bits, but for those of a NaN."""
    a, nan = got.cpu().numpy(), np.isnan(ref)
    return np.array_equal(np.isnan(a), nan) and np.array_equal(a[~nan].view(np.int32), ref[~nan].view(np.int32))


@pytest.mark.parametrize("act", TYPES, ids=str)
@pytest.mark.parametrize("rows,vocab,pitch,out_pitch", [
    (1, 1, None, None), (3, 33, None, None), (2, 4095, 4096, 4100), (2, 4097, None, None), (4, 32003, 32064, 32064),
    (5, 16384, None, None), (1, 70001, 70004, None), (600, 130, 136, None), (520, 16500, None, None), (515, 9001, 9004, 9008)])
def test_sizes(rows, vocab, pitch, out_pitch, act):
    """Pieces of four and of one element, chunks of both sizes, vocabularies that end inside a word and a piece."""
    Case(rows, vocab, act, pitch=pitch, out_pitch=out_pitch).check()


@pytest.mark.parametrize("history,biases,masks", [(0, 0, 0), (40, 0, 0), (0, 40, 0), (0, 0, 2), (40, 0, 1), (0, 9, 1), (5000, 700, 1)])
def test_parts(history, biases, masks):
    Case(6, 5000, torch.bfloat16, history, biases, masks).check()


@pytest.mark.parametrize("rows,vocab,biases", [(3, 4097, 9000), (600, 130, 400), (2, 5000, 760)])
@pytest.mark.parametrize("act", [torch.float16, torch.float32], ids=str)
def test_more_biases_than_a_list_holds(rows, vocab, biases, act):
    """In chunks of both sizes, tokens that are biased many times among them."""
    c = Case(rows, vocab, act, 20, biases, 1, special=True)
    c.check()
    if act is torch.float32:
        ref = c.ref()
        c.out = c.x
        c.out_wide = c.x
        from paper_2609_08450_amd import logits

        assert same(logits.adjust(c.x, c.x, **c.how), ref)


def test_as_many_biases_as_a_list_holds():
    c = Case(3, 1000, biases=1, history=9)
    c.biases = [[((7 * i) % 1000, float(i)) for i in range(n)] for n in (255, 256, 257)]
    c.how["bias_ids"], c.how["bias_starts"] = ragged([[i for i, _ in b] for b in c.biases], torch.int32)
    c.how["bias"] = ragged([[v for _, v in b] for b in c.biases], torch.float32)[0]
    c.check()


def test_special_values():
    """Infinities and zeros of both signs, and NaN: only in tokens that the mask allows does one stay."""
    c = Case(6, 3000, special=True)
    c.check()
    c.x[:, 5:900:7] = float("nan")
    ref = c.ref()
    c.check()
    assert np.isnan(ref).any()
    masked = [r for r, m in enumerate(c.row_mask) if 0 <= m < 3]
    assert masked and all(bool((c.out[r][~torch.from_numpy(c.allowed[c.row_mask[r]]).cuda()] == -torch.inf).all()) for r in masked)


def test_a_mask_that_allows_nothing_and_one_that_allows_all():
    c = Case(4, 1000, masks=2)
    c.allowed[0], c.allowed[1] = False, True
    c.how["mask"] = torch.from_numpy(mask_words(c.allowed)).cuda()
    c.row_mask = [0, 1, 0, -1]
    c.how["row_mask"] = torch.tensor(c.row_mask, dtype=torch.int32).cuda()
    c.check()
    assert bool((c.out[0] == -torch.inf).all())


def test_a_mask_of_each_row_and_wider_masks():
    c = Case(3, 1003, masks=3)
    c.row_mask = [0, 1, 2]
    wide = torch.full((3, 40), -1, dtype=torch.int32, device="cuda")
    words = mask_words(c.allowed)
    wide[:, 2:2 + words.shape[1]] = torch.from_numpy(words).cuda()
    c.check(mask=wide[:, 2:2 + words.shape[1]], row_mask=None)
    c.check(mask=wide[:, 2:], row_mask=None)


def test_one_token_many_times():
    c = Case(2, 5000)
    c.tokens = [[17] * 100000 + [4097] * 3, [4097]]
    c.prompts = [2, 0]
    c.how["tokens"], c.how["token_starts"] = ragged(c.tokens, torch.int32)
    c.how["prompt_lens"] = torch.tensor(c.prompts, dtype=torch.int32).cuda()
    c.check()


def test_without_prompts_and_penalties():
    c = Case(3, 400)
    c.rep[:], c.freq[:], c.pres[:] = 1.0, 0.0, 0.0
    c.check(repetition=None, frequency=None, presence=None)
    c = Case(3, 400)
    c.prompts = [0, 0, 0]
    c.check(prompt_lens=None)
    c.prompts = [-5, 10 ** 9, 0]
    c.how["prompt_lens"] = torch.tensor(c.prompts, dtype=torch.int32).cuda()
    c.check()


def test_empty_lists():
    c = Case(2, 300, history=1, biases=1)
    c.tokens, c.biases = [[], []], [[], []]
    for name, dtype in (("tokens", torch.int32), ("bias_ids", torch.int32)):
        c.how[name] = torch.empty(0, dtype=dtype, device="cuda")
    c.how.update(bias=torch.empty(0, device="cuda"), token_starts=torch.zeros(3, dtype=torch.int64).cuda(),
                 bias_starts=torch.zeros(3, dtype=torch.int64).cuda())
    c.check()
    from paper_2609_08450_amd import logits

    assert logits.adjust(torch.empty((0, 300), device="cuda")).shape == (0, 300)


def test_in_place_and_made():
    from paper_2609_08450_amd import logits

    for pitch in (None, 2052):
        c = Case(4, 2049, pitch=pitch)
        ref = c.ref()
        made = logits.adjust(c.x, **c.how)
        assert same(made, ref)
        around = c.wide.clone()
        assert logits.adjust(c.x, c.x, **c.how) is c.x
        assert same(c.x, ref) and torch.equal(c.wide[:, 2049:], around[:, 2049:])


def test_captured_and_on_other_streams():
    from paper_2609_08450_amd import logits

    c = Case(5, 9000, torch.bfloat16)
    ref = c.ref()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = logits.adjust(c.x, stream=stream, **c.how)
        side.synchronize()
        assert same(got, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits.adjust(c.x, c.out, **c.how)
    for i in range(3):
        c.x.mul_(-1.5)
        eager = logits.adjust(c.x, **c.how)
        graph.replay()
        torch.cuda.synchronize()
        assert same(c.out, c.ref()) and same(eager, c.ref()), i


def test_a_top_k_reads_the_rows():
    """The chain: penalties, mask, then the selection of the candidates of each row."""
    from paper_2609_08450_amd import logits, topk

    c = Case(8, 32003, torch.bfloat16, out_pitch=32064)
    c.check()
    rows = torch.full((8, 32064), -torch.inf, device="cuda")
    logits.adjust(c.x, rows[:, :32003], **c.how)
    idx, val = topk.TopK(8, 64)(rows, torch.arange(8).cuda() * 32064, torch.full((8,), 32003, dtype=torch.int32).cuda())
    ref = torch.from_numpy(c.ref())
    want = torch.sort(ref, 1, descending=True).values[:, :64]
    assert torch.equal(torch.sort(val.cpu(), 1, descending=True).values, want)
    assert torch.equal(ref.gather(1, idx.cpu().long()), val.cpu())
