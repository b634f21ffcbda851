"""The list of kept tokens, and the cache moved together, against their definitions."""
import numpy as np
import pytest
import torch

from tests.paged_util import Setup, assert_attention, attention
from tests.serve_util import compacted, kept

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def run_keep(idx, lens, first, last, base=0, width=None, weights=None):
    """Lists from keep(), checked against the definition, and the weights' rows."""
    from paper_2609_08450_amd import evict

    n, K = len(lens), len(idx[0]) if idx else 0
    width = first + K + last if width is None else width
    out = torch.full((n, width), 77, dtype=torch.int32, device="cuda")
    counts = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    t = torch.tensor(idx, dtype=torch.int32).reshape(n, K).cuda()
    how = {}
    if weights is not None:
        pitch = weights.shape[1]
        how = dict(weights=weights, weight_offsets=torch.arange(n).cuda() * pitch)
    evict.keep(t, torch.tensor(lens, dtype=torch.int32).cuda(), first, last, out, counts, base=base, **how)
    ref = kept(idx, lens, first, last, base)
    assert counts.tolist() == [len(x) for x in ref]
    assert out.tolist() == [x + [-1] * (width - len(x)) for x in ref]
    return ref, out, counts


KEEPS = [  # lengths, K, first, last, base
    ([10], 3, 0, 0, 0), ([0, 1, 2, -5], 4, 1, 1, 0), ([31, 32, 33, 64, 1000], 8, 2, 3, 2), ([5000, 7], 700, 4, 500, 4),
    ([100], 0, 30, 30, 0), ([100], 0, 0, 0, 0), ([40], 5, 100, 3, 0), ([40], 5, 3, 100, 0), ([70000], 2048, 64, 448, 64),
    ([600000], 5000, 10, 90, 10), ([524288, 524289, 1048577], 300, 1, 2, 1), ([3000] * 40, 64, 4, 60, 4),
]


@pytest.mark.parametrize("lens,K,first,last,base", KEEPS, ids=str)
def test_keep(lens, K, first, last, base):
    """Tokens given twice, below 0, past the length, inside the first and the last ones; weights moved along."""
    g = np.random.default_rng(K)
    idx = [g.integers(-3, max(L, 1) + 5, K).tolist() for L in lens]
    pitch = max(max(lens), 1) + 9
    weights = torch.rand((len(lens), pitch), generator=torch.Generator().manual_seed(K)).cuda()
    before = weights.cpu()
    ref, _, _ = run_keep(idx, lens, first, last, base, weights=weights)
    run_keep(idx, lens, first, last, base, width=first + K + last + 13)
    after = weights.cpu()
    for r, L in enumerate(lens):
        L = max(L, 0)
        assert torch.equal(after[r, :len(ref[r])], before[r, ref[r]])
        assert bool((after[r, len(ref[r]):L] == 0).all()) and torch.equal(after[r, L:], before[r, L:])


def test_keep_at_the_end_of_32_bits():
    """The longest request that is counted: the bits go through LDS in rounds."""
    L = 2 ** 31 - 1
    run_keep([[5, L - 1, L - 2, 2 ** 30, 2 ** 31 - 100, 5, -1]], [L], 2, 3)
    run_keep([[2 ** 31 - 1, 2 ** 31 - 4, 0]], [L], 0, 0, base=2)


def moved(s, lists, where="", table=None, stream=None):
    """compact() of s's cache by these lists against the definition; codes that it must not touch too."""
    from paper_2609_08450_amd import evict

    width = max([1, *map(len, lists)])
    t = torch.tensor([x + [-1] * (width - len(x)) for x in lists], dtype=torch.int32).cuda()
    counts = torch.tensor([len(x) for x in lists], dtype=torch.int32).cuda()
    dtype, sides = s.k.dtype, [("k", "ks")] + ([("v", "vs")] if s.v is not None else [])
    rows = s.table.tolist()
    ref = {}
    for codes, scale in sides:
        x = getattr(s, codes)
        ref[codes] = compacted(x.float().cpu().numpy().astype(np.float64), getattr(s, scale).cpu().numpy(), rows, lists,
                               s.page, dtype)
    before = {c: getattr(s, c).view(torch.uint8).cpu() for c, _ in sides}
    evict.compact(s.cache(), s.table, t, counts, stream=stream)
    torch.cuda.synchronize()
    for codes, scale in sides:
        got = getattr(s, codes)
        want, ws = ref[codes]
        assert torch.equal(getattr(s, scale).cpu(), torch.from_numpy(ws)), f"{where}: {scale}"
        x = got.float().cpu().numpy()
        same = (x == want) | (np.isnan(x) & np.isnan(want))
        assert same.all(), f"{where}: {codes} {np.argwhere(~same)[0].tolist()}, {int((~same).sum())} differ"
        # what was NaN has its bits still: nothing outside the lists is written
        nan = torch.from_numpy(np.isnan(want))
        assert torch.equal(got.view(torch.uint8).cpu()[nan], before[codes][nan])


def some(lens, keep, seed=0):
    g = np.random.default_rng(seed)
    return [sorted(g.choice(L, min(k, L), replace=False).tolist()) for L, k in zip(lens, keep)]


SIZES = [  # lengths, kept, page, kv, dim
    ([1], [1], 16, 1, 64), ([2, 0, 17], [1, 0, 5], 16, 2, 64), ([200, 33, 400], [60, 33, 399], 16, 2, 128),
    ([1000], [129], 32, 3, 64), ([700, 1300], [500, 64], 64, 2, 128), ([900], [256], 128, 1, 128),
    ([2500], [1100], 64, 1, 256), ([3000, 600], [1030, 257], 256, 1, 256), ([5000], [3000], 16, 1, 64),
    ([600], [300], 256, 2, 64), ([4000], [2048], 128, 8, 64), ([513], [511], 32, 1, 256),
]


@pytest.mark.parametrize("code", [E4M3, torch.int8], ids=str)
@pytest.mark.parametrize("lens,keep,page,kv,dim", SIZES, ids=str)
def test_compact(lens, keep, page, kv, dim, code):
    s = Setup(lens, [1] * len(lens), page=page, kv=kv, heads=kv, dim=dim, code=code, seed=page + dim).cuda()
    moved(s, some(lens, keep))


@pytest.mark.parametrize("code", [E4M3, torch.int8], ids=str)
@pytest.mark.parametrize("page,dim", [(16, 64), (256, 64), (32, 128), (256, 128), (128, 256), (256, 256)], ids=str)
def test_compact_of_many_requests(page, dim, code):
    """64 requests of 4 heads, K and V: 512 workgroups, which have 8 waves each where a page's codes of a head are at most
    32768 bytes (a round is then one page at the largest, several at smaller ones).  Most are short, some take several rounds."""
    lens = [40 + 3 * i for i in range(60)] + [1500, 1300, 1100, 2 * page + 1]
    keep = [1 + (11 * n) % 90 for n in lens[:60]] + [1290, 640, 513, page + 1]
    s = Setup(lens, [1] * 64, page=page, kv=4, heads=4, dim=dim, code=code, seed=page + dim).cuda()
    moved(s, some(lens, keep))


def test_compact_of_power_of_two_scales():
    """As the store leaves e4m3 pages."""
    s = Setup([800, 90], [1, 1], page=32, kv=2, heads=2, dim=64)
    s.ks, s.vs = (torch.exp2(torch.round(torch.log2(x))) for x in (s.ks, s.vs))
    moved(s.cuda(), some([800, 90], [300, 20]))


@pytest.mark.parametrize("code", [E4M3, torch.int8], ids=str)
def test_what_stays_is_not_touched(code):
    """Nothing evicted, a prefix, a tail cut off, a single gap at every place near a page's end."""
    for lists in ([list(range(100))], [list(range(64))], [[]], [list(range(70))], [[i for i in range(100) if i != 15]],
                  [[i for i in range(100) if i != 16]], [[i for i in range(100) if i != 99]], [[99]], [list(range(16)) + [99]],
                  [list(range(1, 100))]):
        s = Setup([100], [1], page=16, kv=2, heads=2, dim=64, code=code).cuda()
        moved(s, lists, where=str(lists[0][:3]) + str(len(lists[0])))


@pytest.mark.parametrize("code", [E4M3, torch.int8], ids=str)
def test_extreme_scales_and_codes(code):
    """Scales far apart in one page, 0, the least ones; codes of 0 alone, of the type's largest and least."""
    s = Setup([512], [1], page=16, kv=2, heads=2, dim=64, code=code, seed=3)
    pages = s.table[0].long()
    s.ks[pages[::3]] *= 2.0 ** 20
    s.ks[pages[1::5], 0] = 0.0
    s.ks[pages[2::7]] = 2.0 ** -100
    s.ks[pages[3]], s.ks[pages[4]] = 1e-38, 1e30
    if code is torch.int8:
        s.k[pages[6]], s.v[pages[7]] = -128, 127
    else:
        s.k.view(torch.uint8)[pages[6]] = 0x01
        s.v.view(torch.uint8)[pages[7]] = 0x7E
    s.k[pages[8:12]] = torch.zeros((4, 2, 16, 64)).to(code)
    moved(s.cuda(), some([512], [200], seed=5))


@pytest.mark.parametrize("code", [E4M3, torch.int8], ids=str)
def test_codes_of_zero_under_scales_of_any_size(code):
    """0 stays 0 beside the least scales, and one that is 2^20 to 2^200 times as large."""
    for big in (2.0 ** -80, 1.0, 3e38):
        s = Setup([64], [1], page=16, kv=1, heads=1, dim=64, code=code, seed=6)
        pages = s.table[0].long()
        s.k[pages[1]] = torch.zeros((1, 16, 64)).to(code)
        s.ks[:] = 2.0 ** -100
        s.ks[pages[1]] = big
        moved(s.cuda(), [[0, 2, 16, 17, 30, 40, 50, 60, 61, 62]], where=str(big))


def test_scales_many_times_the_new_one():
    """What had the old scale's large codes is gone: codes of 1, 2, .. grow up to 127 fold, and round as exactly."""
    g = np.random.default_rng(8)
    for k in range(12):
        s = Setup([640], [1], page=16, kv=1, heads=1, dim=64, code=torch.int8, seed=k)
        pages = s.table[0].long()
        small = torch.from_numpy(g.integers(-(k + 1), k + 2, (40, 1, 16, 64)).astype(np.int8))
        s.k[pages] = small
        s.ks[pages] = torch.from_numpy(g.uniform(0.5, 1.0 + 3 * k, (40, 1)).astype(np.float32))
        moved(s.cuda(), some([640], [300], seed=k), where=str(k))


def test_ties_round_to_even():
    """Scales whose quotients are halves: exact ties, and quotients next to one."""
    s = Setup([64], [1], page=16, kv=1, heads=1, dim=64, code=torch.int8)
    pages = s.table[0].long()
    s.k[pages[0]] = 127
    s.k[pages[1:]] = torch.arange(-96, 96, dtype=torch.int8).view(3, 1, 1, 64).expand(3, 1, 16, 64)
    for big, small in ((127.0, 63.5), (254.0, 1.0), (1.0, 0.5 + 2.0 ** -24), (1.0, 0.5 - 2.0 ** -25), (3.0, 1.5), (1.0, 0.1)):
        t = Setup([64], [1], page=16, kv=1, heads=1, dim=64, code=torch.int8)
        t.k, t.table = s.k.clone(), s.table
        t.ks[:] = small
        t.ks[pages[0]] = big
        moved(t.cuda(), [[1, *range(17, 64, 3)]], where=str((big, small)))


def test_keys_alone_and_strided_caches():
    from paper_2609_08450_amd import paged

    s = Setup([300, 90], [1, 1], page=32, kv=2, heads=2, dim=64, values=False).cuda()
    layers = torch.zeros((s.n_pages, 3, 2, 32, 64), dtype=torch.uint8, device="cuda")
    layers[:, 1] = s.k.view(torch.uint8)
    scales = torch.ones((s.n_pages, 3, 2), device="cuda")
    scales[:, 1] = s.ks
    s.k, s.ks = layers.view(E4M3)[:, 1], scales[:, 1]
    s.cache = lambda: paged.PagedCache.of(s.k, s.ks)
    moved(s, some([300, 90], [120, 17]))
    assert bool((layers[:, 0] == 0).all()) and bool((layers[:, 2] == 0).all())
    assert bool((scales[:, 0] == 1).all()) and bool((scales[:, 2] == 1).all())


@pytest.mark.parametrize("code", [E4M3, torch.int8], ids=str)
def test_pages_outside_the_cache(code):
    s = Setup([300, 200], [1, 1], page=16, kv=1, heads=1, dim=64, code=code)
    s.table[0, 3], s.table[0, 15], s.table[1, 0], s.table[1, 9] = -1, s.n_pages, 2 ** 31 - 1, -2 ** 31
    moved(s.cuda(), some([300, 200], [100, 90]))


def test_counts_and_lists_past_the_table():
    """A count beyond the list's width, the table's, or below 0, and numbers past the table: nothing is read or written there."""
    from paper_2609_08450_amd import evict

    s = Setup([64, 64, 64], [1, 1, 1], page=16, kv=1, heads=1, dim=64, code=torch.int8).cuda()
    before = s.k.clone()
    t = torch.tensor([[5, 7, 10 ** 6, 2 ** 31 - 1], [3, -1, -5, 63], [1, 2, 3, 4]], dtype=torch.int32).cuda()
    evict.compact(s.cache(), s.table, t, torch.tensor([9, 4, -1], dtype=torch.int32).cuda())
    first = s.table[:, 0].long()
    assert bool((s.k[first[0], :, 2:4] == 0).all()) and torch.equal(s.k[first[0], :, 4:], before[first[0], :, 4:])
    assert torch.equal(s.k[s.table[2].long()], before[s.table[2].long()])
    assert torch.equal(s.k[s.table[:, 1:].long()], before[s.table[:, 1:].long()])


def test_attention_over_what_is_kept():
    """keep, compact, then attend: what the rows see is the kept tokens' values."""
    from paper_2609_08450_amd import paged

    s = Setup([900, 400], [1, 1], page=32, kv=2, heads=8, dim=64).cuda()
    idx = [list(range(3, 800, 9)) + [3, -1], [5] * 91]
    idx[1] += [7] * (len(idx[0]) - 91)
    lists, t, counts = run_keep(idx, [900, 400], 4, 60)
    moved(s, lists)
    s.row_lengths = counts
    lse = torch.empty((2, 8), device="cuda")
    out = paged.attend(s.cache(), s.q, s.table, s.row_starts, counts, s.scale, lse=lse)
    assert_attention(out, lse, attention(s))


def test_captured_and_on_other_streams():
    from paper_2609_08450_amd import evict

    def setup():
        return Setup([700, 300], [1, 1], page=32, kv=2, heads=2, dim=128, code=torch.int8, seed=4).cuda()

    lens, offsets = torch.tensor([700, 300], dtype=torch.int32).cuda(), torch.tensor([0, 700]).cuda()
    idx = torch.tensor([[650, 3, 77, 500, 2], [8, 120, -1, 4, 250]], dtype=torch.int32).cuda()

    def chain(s, w, out, counts, stream=None):
        evict.keep(idx, lens, 40, 30, out, counts, weights=w, weight_offsets=offsets, stream=stream)
        evict.compact(s.cache(), s.table, out, counts, stream=stream)

    def state(s):
        return s, torch.rand(1000, generator=torch.Generator().manual_seed(1)).cuda(), \
            torch.empty((2, 75), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")

    def same(a, b):
        return all(torch.equal(x, y) for x, y in zip((a[0].k, a[0].v, a[0].ks, a[0].vs, *a[1:]),
                                                     (b[0].k, b[0].v, b[0].ks, b[0].vs, *b[1:])))

    ref = state(setup())
    chain(*ref)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        x = state(setup())
        torch.cuda.synchronize()
        chain(*x, stream=stream)
        torch.cuda.synchronize()
        assert same(x, ref)
    x, fresh = state(setup()), state(setup())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(*x)
    for i in range(3):
        for a, b in zip((x[0].k, x[0].v, x[0].ks, x[0].vs, x[1]), (fresh[0].k, fresh[0].v, fresh[0].ks, fresh[0].vs, fresh[1])):
            a.copy_(b)
        other = state(setup())
        chain(*other)
        graph.replay()
        torch.cuda.synchronize()
        assert same(x, ref) and same(other, ref), i


def test_far_pages():
    """Codes past 2^32 bytes."""
    from paper_2609_08450_amd import evict, paged

    n_pages = 2 ** 32 // (16 * 64) + 64
    k = torch.zeros((n_pages, 1, 16, 64), dtype=torch.int8, device="cuda")
    ks = torch.ones((n_pages, 1), device="cuda")
    at = torch.tensor([n_pages - 1, 3, n_pages - 2, n_pages - 5])
    x = torch.randint(-127, 128, (4, 1, 16, 64), generator=torch.Generator().manual_seed(2)).to(torch.int8)
    x[0, 0, 5] = x[1, 0, 0] = x[2, 0, 7] = x[3, 0, 15] = 127
    k[at.cuda()] = x.cuda()
    evict.compact(paged.PagedCache.of(k, ks), at.int().cuda()[None],
                  torch.tensor([[5, 16, 39, 63]], dtype=torch.int32).cuda(), torch.tensor([4], dtype=torch.int32).cuda())
    got = k[at.cuda()].cpu()
    assert torch.equal(got[0, 0, :4], torch.stack([x[0, 0, 5], x[1, 0, 0], x[2, 0, 7], x[3, 0, 15]]))
    assert torch.equal(got[0, 0, 4:], x[0, 0, 4:]) and torch.equal(got[1:], x[1:])
