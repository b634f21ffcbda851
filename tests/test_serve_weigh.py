"""Accumulated attention weights against their definition in 64 bits."""
import math

import pytest
import torch

from tests.paged_util import Setup
from tests.serve_util import weighed

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def lse_of(s, seed=0):
    """That of each row's softmax, by the definition; -inf where a row sees nothing."""
    out = torch.full((s.n_rows, s.heads), -math.inf)
    cap = s.table.shape[1] * s.page
    G = s.heads // s.kv
    for i in range(s.n_rows):
        r, L = int(s.row_request[i]) if i < len(s.row_request) else -1, min(max(int(s.row_lengths[i]), 0), cap)
        if r < 0 or L == 0:
            continue
        k, there = s.tokens("k", r, L)
        if not bool(there.any()):
            continue
        q = s.q[i].double().view(s.kv, G, s.dim)
        x = s.scale * torch.matmul(q, k[:, there].transpose(1, 2))
        out[i] = torch.logsumexp(x, -1).reshape(s.heads).float().cpu()
    return out.to(s.q.device)


def check(s, lse=None, where="", workspace=None, table=None, **how):
    from paper_2609_08450_amd import evict

    lse = lse_of(s) if lse is None else lse
    n = len(s.row_starts) - 1
    sums, bounds, held = weighed(s, lse, how.get("scale"))
    room = max([1, *map(len, sums)]) + 5
    g = torch.Generator().manual_seed(9)
    before = torch.rand((n, room), generator=g).cuda()
    # rows of weights in any order, at any offset
    order = torch.randperm(n, generator=g).cuda()
    weights, offsets = before.clone(), order * room + (1 if n * room > 1 else 0)
    flat = torch.cat([torch.zeros(1, device="cuda"), weights.flatten()])
    evict.weigh(s.cache(), s.q, lse, s.table, s.row_starts, s.row_lengths, how.get("scale", s.scale), flat, offsets,
                workspace=workspace, stream=how.get("stream"))
    torch.cuda.synchronize()
    got, seen = flat[1:].view(n, room), 0
    for r in range(n):
        a, b, L = got[order[r]], before[order[r]].double(), len(sums[r])
        assert torch.equal(a[L:].double(), b[L:]), f"{where}: past the tokens of request {r}"
        if L == 0:
            continue
        assert torch.equal(a[:L].double()[~held[r]], b[:L][~held[r]]), f"{where}: tokens outside the cache, request {r}"
        ref = b[:L] + sums[r]
        tol = bounds[r] + 2.0 ** -22 * ref.abs()
        # a row that sees an entry that is NaN (one past its request's tokens) has an lse that is NaN, and so its tokens' sums
        nan = torch.isnan(ref) & held[r]
        assert torch.equal(torch.isnan(a[:L]), nan), f"{where}: NaN, request {r}"
        off = ((a[:L].double() - ref).abs() - tol)[held[r] & ~nan]
        assert not bool((off > 0).any()) and not bool(torch.isinf(a).any()), f"{where}: request {r}, by {float(off.max()):.3g}"
        seen += int((sums[r] > 0).sum())
    return seen


SIZES = [  # lengths, rows, page, kv, heads, dim
    ([1], [1], 16, 1, 1, 64), ([1, 0, 17], [1, 0, 1], 16, 2, 2, 64), ([255, 256, 257, 1025], [1, 1, 1, 1], 16, 4, 8, 64),
    ([700, 33], [1, 1], 64, 2, 16, 128), ([3000], [1], 256, 1, 16, 128), ([513], [1], 32, 8, 32, 256),
    ([90, 2049], [1, 1], 128, 1, 40, 128), ([300], [1], 64, 1, 130, 64), ([65], [1], 64, 1, 70, 256),
    ([400, 77], [3, 2], 16, 2, 6, 128), ([600, 5, 1200], [37, 5, 130], 32, 2, 6, 64), ([300], [300], 64, 1, 4, 128),
    ([97, 130, 513], [33, 130, 1], 16, 4, 4, 256), ([1500], [200], 128, 2, 16, 128), ([40] * 70, [1] * 70, 16, 1, 3, 64),
]


@pytest.mark.parametrize("lens,rows,page,kv,heads,dim", SIZES, ids=str)
@pytest.mark.parametrize("code,act", [(E4M3, torch.bfloat16), (torch.int8, torch.float16)], ids=str)
def test_sizes(lens, rows, page, kv, heads, dim, code, act):
    s = Setup(lens, rows, page=page, kv=kv, heads=heads, dim=dim, code=code, act=act, seed=len(lens), values=False)
    assert check(s.cuda()) == sum(lens)


@pytest.mark.parametrize("code,act", [(E4M3, torch.float16), (torch.int8, torch.bfloat16)], ids=str)
def test_other_types(code, act):
    check(Setup([130, 600], [2, 40], page=32, kv=2, heads=8, dim=64, code=code, act=act, values=False).cuda())


def test_rows_that_see_anything():
    """Lengths in no order, none, past the table and negative: a request's rows need not be a causal block."""
    seen = [5, 0, 300, 17, 64, 1, 299, 10 ** 6, -4, 300, 33, 0]
    for heads in (4, 32):
        s = Setup([300, 300], [7, 5], page=16, kv=2, heads=heads, dim=64, seen=seen, values=False).cuda()
        check(s, where=str(heads))
    # the table's end is the requests' here, so that every token that a row can see is one
    s = Setup([304, 304], [7, 5], page=16, kv=2, heads=32, dim=64, seen=seen, values=False).cuda()
    assert check(s) == 300 + 304  # the longest of each request's rows
    seen = (seen * 40)[:400]
    s = Setup([304, 304], [390, 10], page=16, kv=2, heads=8, dim=64, seen=seen, values=False).cuda()
    assert check(s, where="many") == 608


def test_rows_without_a_softmax():
    """An lse of -inf adds nothing, whatever its queries hold."""
    for rows in ([4, 1], [70, 40]):
        s = Setup([200, 90], rows, page=16, kv=2, heads=8, dim=128, values=False).cuda()
        lse = lse_of(s)
        lse[1], lse[3, 5] = -math.inf, -math.inf
        s.q[1], s.q[3, 5] = math.nan, math.inf
        clean = s.q.clone()
        clean[1], clean[3, 5] = 0.0, 0.0
        held, s.q = s.q, clean
        sums = weighed(s, lse)[0]
        s.q = held
        from paper_2609_08450_amd import evict

        w = torch.zeros((2, 200), device="cuda")
        evict.weigh(s.cache(), s.q, lse, s.table, s.row_starts, s.row_lengths, s.scale, w,
                    torch.tensor([0, 200], device="cuda"))
        for r in range(2):
            assert bool(torch.isfinite(w[r]).all())
            assert bool(((w[r, :len(sums[r])].double() - sums[r]).abs() <= 1e-3 * sums[r] + 1e-30).all())


@pytest.mark.parametrize("lens,rows,heads,dim", [
    ([100, 90], [1, 1], 8, 64), ([100] * 300, [1] * 300, 4, 64), ([100, 90], [4, 1], 8, 128), ([100, 600], [70, 40], 8, 128),
    ([100, 600], [30, 40], 16, 256), ([600], [40], 2, 64)], ids=str)
def test_rows_without_a_softmax_see_keys_that_are_nan(lens, rows, heads, dim):
    """An lse of -inf adds nothing, whatever the keys hold: rows that see codes behind a request's tokens, NaN here, by
    themselves, among others of their window, and as all of a window."""
    s = Setup(lens, rows, page=16, kv=2, heads=heads, dim=dim, values=False).cuda()
    cap, starts = s.table.shape[1] * 16, s.row_starts.tolist()
    lse = lse_of(s)
    for r, n in enumerate(lens):
        # the pages' last tokens are what nobody has stored
        s.row_lengths[starts[r]] = -(-n // 16) * 16 if n % 16 else min(n, cap)
        lse[starts[r]] = -math.inf
    check(s, lse)
    for r, n in enumerate(lens):
        s.row_lengths[starts[r]:starts[r + 1]] = -(-n // 16) * 16
    lse[:] = -math.inf
    check(s, lse)


@pytest.mark.parametrize("rows", [[1, 1], [40, 30]], ids=str)
def test_softmaxes_of_any_size(rows):
    """Finite ones up to the largest FP32 number: exp of what is left is 0, or past every number."""
    from paper_2609_08450_amd import evict

    s = Setup([100, 333], rows, page=16, kv=2, heads=8, dim=64, values=False).cuda()
    lse = lse_of(s)
    for i, z in enumerate((1e8, 1.1e9, 1e10, 3.3e10, 7.7e15, 1e20, 1.7e30, 2.4e38, 2.36e38, 3.4e38)):
        far = torch.full_like(lse, z) * (1 + 2.0 ** -20 * torch.rand(lse.shape, generator=torch.Generator().manual_seed(i)).cuda())
        far = far.clamp(max=torch.finfo(torch.float32).max)
        check(s, far, where=str(z))
        few = lse.clone()
        few[:, 3], few[-1] = far[:, 3], far[-1]
        check(s, few, where=f"{z} among others")
        w = torch.zeros((2, 400), device="cuda")
        evict.weigh(s.cache(), s.q, -far, s.table, s.row_starts, s.row_lengths, s.scale, w, torch.tensor([0, 400]).cuda())
        for r in range(2):
            seen = int(s.row_lengths[s.row_starts[r]:s.row_starts[r + 1]].max())
            assert bool((w[r, :seen] == math.inf).all()) and not bool(w[r, seen:].any()), z


def test_pages_outside_the_cache():
    for rows in ([1, 1], [50, 30]):
        s = Setup([100, 333], rows, page=16, kv=2, heads=4, dim=64, values=False)
        s.table[0, 2], s.table[1, 5], s.table[1, 20] = -1, s.n_pages, 2 ** 31 - 1
        check(s.cuda(), where=str(rows))
    s = Setup([20], [1], page=16, kv=1, heads=1, dim=64, values=False)
    s.table[:] = -7
    check(s.cuda())


def test_rows_of_no_request():
    """Rows before the first request's, between a falling pair of starts, and past the last."""
    s = Setup([60, 70], [3, 4], page=16, kv=1, heads=4, dim=64, values=False)
    s.row_starts = torch.tensor([2, 3, 6], dtype=torch.int32)
    s.row_request = torch.tensor([-1, -1, 0, 1, 1, 1, -1], dtype=torch.int32)
    s.row_lengths = torch.tensor([50, 50, 60, 68, 69, 70, 40], dtype=torch.int32)
    check(s.cuda())
    for starts in ([5, 2, 7], [-3, 4, 100]):
        s.row_starts = torch.tensor(starts, dtype=torch.int32).cuda()
        at = [min(max(x, 0), 7) for x in starts]
        s.row_request = torch.tensor([0 if at[0] <= i < at[1] else 1 if at[1] <= i < at[2] else -1 for i in range(7)],
                                     dtype=torch.int32).cuda()
        check(s, where=str(starts))


def test_strided_queries_and_caches():
    """Queries in a projection's output, a layer's slice of the pages, a table's first columns."""
    from paper_2609_08450_amd import paged

    for rows in ([1, 1], [64, 9]):
        s = Setup([150, 90], rows, page=32, kv=2, heads=4, dim=64, values=False).cuda()
        wide = torch.zeros((s.n_rows, 9, 64), dtype=s.act, device="cuda")
        wide[:, 2:6] = s.q
        s.q = wide[:, 2:6]
        layers = torch.zeros((s.n_pages, 3, 2, 32, 64), dtype=torch.uint8, device="cuda")
        layers[:, 1] = s.k.view(torch.uint8)
        scales = torch.full((s.n_pages, 3, 2), math.nan, device="cuda")
        scales[:, 1] = s.ks
        s.cache = lambda: paged.PagedCache.of(layers.view(E4M3)[:, 1], scales[:, 1])
        table = torch.full((2, s.table.shape[1] + 4), -1, dtype=torch.int32, device="cuda")
        table[:, :s.table.shape[1]] = s.table
        s.table = table[:, :s.table.shape[1]]
        check(s)


def test_scale_zero_and_no_heads_in_common():
    s = Setup([77], [2], page=16, kv=1, heads=3, dim=64, values=False).cuda()
    check(s, lse=torch.full((2, 3), 1.5, device="cuda"), scale=0.0)


@pytest.mark.parametrize("rows", [[1, 1], [40, 30]], ids=str)
def test_the_least_scales(rows):
    """Below FP32's least normal number a scale has few bits: what its rounding leaves is then no factor of the weights."""
    s = Setup([100, 333], rows, page=16, kv=2, heads=8, dim=64, values=False).cuda()
    for s.scale in (1.4e-45, 2e-45, 3e-44, 1e-42, 7e-40, 1.17e-38, 1e-37, 1e-30):
        check(s, where=str(s.scale))


def test_weights_of_a_softmax_sum_to_one_a_row_and_head():
    """With attend's lse: every row and head gives one away."""
    from paper_2609_08450_amd import evict, paged

    for rows in ([1, 1, 1], [20, 300, 1]):
        s = Setup([900, 5000, 64], rows, page=64, kv=2, heads=8, dim=128).cuda()
        cache, lse = s.cache(), torch.empty((s.n_rows, 8), device="cuda")
        paged.attend(cache, s.q, s.table, s.row_starts, s.row_lengths, s.scale, lse=lse)
        w = torch.zeros((3, 5000), device="cuda")
        evict.weigh(cache, s.q, lse, s.table, s.row_starts, s.row_lengths, s.scale, w, torch.arange(3).cuda() * 5000)
        total = w.double().sum(1).cpu()
        want = torch.tensor(rows, dtype=torch.float64) * 8
        # attend's lse and these exponents: 2^-15 of (1 + |lse|) as its test allows, |lse| below 40
        assert bool(((total - want).abs() <= want * 41 * 2.0 ** -15).all()), total


def test_repeats_to_the_bit_captured_and_on_other_streams():
    from paper_2609_08450_amd import evict

    for rows in ([1, 1], [150, 61]):
        s = Setup([3000, 700], rows, page=32, kv=2, heads=8, dim=64, values=False).cuda()
        cache, lse, offsets = s.cache(), lse_of(s), torch.tensor([0, 3000]).cuda()
        args = (s.q, lse, s.table, s.row_starts, s.row_lengths, s.scale)

        def eager(stream=None, workspace=None):
            w = torch.full((3700,), 0.5, device="cuda")
            torch.cuda.synchronize()
            evict.weigh(cache, *args, w, offsets, stream=stream, workspace=workspace)
            torch.cuda.synchronize()
            return w

        ref = eager()
        need = evict.workspace_size(cache, s.n_rows, 2, 8)
        dirty = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        for got in (eager(), eager(side), eager(side.cuda_stream), eager(workspace=dirty), eager(workspace=dirty)):
            assert torch.equal(got, ref)
        w, graph = torch.zeros(3700, device="cuda"), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            evict.weigh(cache, *args, w, offsets)
        for i in range(3):
            eager()
            w.fill_(0.5)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(w, ref), i


@pytest.mark.parametrize("lens,rows", [
    ([900, 300, 513, 1400, 40, 77], [1, 32, 33, 500, 0, 2]),   # few tokens: every request in windows
    ([2040, 900, 300, 513, 1400, 40, 77] + [100] * 57, [3, 1, 32, 33, 500, 0, 2] + [1] * 57),  # rows x heads of 256 and 264
    ([600] + [20] * 63, [60] + [0] * 63),                      # no more rows than requests: one has all of them
    ([700, 50, 31], [20, 4, 5]), ([40000], [25]), ([40000, 9], [31, 1]),  # rows x heads of 256 in all
], ids=str)
@pytest.mark.parametrize("kv,dim", [(2, 64), (8, 128), (1, 256)], ids=str)
def test_requests_of_few_and_of_many_rows(lens, rows, kv, dim):
    """Each kind is a kernel's own, in one call where requests are of both; waves that have the same tokens."""
    s = Setup(lens, rows, page=32, kv=kv, heads=8, dim=dim, values=False).cuda()
    assert check(s) == sum(n for n, r in zip(lens, rows) if r)


ENDS = [1, 0, 2, 63, 64, 65, 127, 255, 256, 257, 300, 511, 512, 513, 700, 767, 768, 769, 900, 1023, 1024, 1025, 1279, 1280,
        1281, 1500, 1793, 2047, 2048, 2049, 2100, 3073]


@pytest.mark.parametrize("width", [8192, 16384])
@pytest.mark.parametrize("kv,heads,dim,code", [(5, 160, 64, E4M3), (1, 130, 64, torch.int8), (4, 80, 256, torch.int8),
                                               (2, 8, 128, E4M3)], ids=str)
def test_tables_far_wider_than_the_requests(kv, heads, dim, code, width):
    """64 requests under a table of 8192 and of 16384 tokens: workgroups of two and of four tiles, lengths that end at
    every one's edges, and several passes over the queries' columns.  Then with two rows to some requests, which
    go to either kernel by their heads."""
    for rows in ([1] * 64, [2, 1, 3, 2, 1, 1, 2, 0] + [1] * 20 + [3] + [1] * 35):
        s = Setup((ENDS * 2)[:len(rows)], rows, page=16, kv=kv, heads=heads, dim=dim, code=code, values=False)
        table = torch.full((len(rows), width // 16), -1, dtype=torch.int32)
        table[:, :s.table.shape[1]] = s.table
        s.table = table
        s = s.cuda()
        assert check(s, where=str(rows[:8])) == sum(n for n, r in zip(s.lens, rows) if r)


@pytest.mark.parametrize("kv,heads,dim,lens,rows", [
    (1, 300, 64, [300, 520], [3, 2]), (1, 257, 64, [33], [4]), (2, 1400, 128, [300], [2]), (1, 130, 256, [300, 40], [5, 1]),
    (2, 400, 256, [513, 257], [3, 4]), (1, 129, 256, [90], [2])], ids=str)
def test_more_heads_of_a_cache_head_than_a_window(kv, heads, dim, lens, rows):
    """Windows of a part of one row's heads, the last part smaller than the others."""
    s = Setup(lens, rows, page=32, kv=kv, heads=heads, dim=dim, values=False).cuda()
    assert check(s) == sum(lens)


def test_more_requests_than_a_round_of_the_plan():
    """Of 560 requests, a few with more rows than the kernel of few rows takes, at the round's edges among them."""
    rows = [17 if r in (0, 99, 511, 512, 559) else 0 if r % 5 == 2 else 1 for r in range(560)]
    s = Setup([(7 * r) % 90 + 20 for r in range(560)], rows, page=16, kv=1, heads=16, dim=64, values=False).cuda()
    assert sum(rows) <= 560  # read by rows
    check(s)
    rows = [r + 40 * (r == 17) for r in rows]
    s = Setup([(7 * r) % 90 + 60 for r in range(560)], rows, page=16, kv=1, heads=16, dim=64, values=False).cuda()
    assert sum(rows) > 560
    check(s)


def test_more_parts_than_the_workspace_holds():
    """Windows add up in one part then; beside them a request of one window, one without rows and one whose windows
    are a single piece."""
    from paper_2609_08450_amd import evict

    # (one head is compared at a time: the others have an lse of -inf but for the first and the last)
    s = Setup([20000, 900, 50, 700], [1280, 3, 0, 40], page=256, kv=8, heads=128, dim=64, values=False).cuda()
    steps = sum(-(-L // 256) * -(-n * 16 // 256) * 8 for L, n in zip(s.lens, (1280, 3, 0, 40)))
    assert steps > 49152
    lse, total, bound = torch.full((s.n_rows, 128), -math.inf, device="cuda"), {}, {}
    for r in (0, 1, 3):
        a, b, L = int(s.row_starts[r]), int(s.row_starts[r + 1]), s.lens[r]
        k, there = s.tokens("k", r, L)
        assert bool(there.all())
        seen = torch.arange(L, device="cuda") < s.row_lengths[a:b, None]
        for h in (0, 77, 127):
            q = s.q[a:b, h].double()
            x = s.scale * torch.matmul(q, k[h // 16].t())
            x.masked_fill_(~seen, -math.inf)
            lse[a:b, h] = torch.logsumexp(x, 1).float()
            z = lse[a:b, h, None].double()
            p = torch.exp(x - z)
            size = s.scale * torch.matmul(q.abs(), k[h // 16].abs().t())
            total[r] = total.get(r, 0) + p.sum(0)
            x.masked_fill_(~seen, 0.0)
            bound[r] = bound.get(r, 0) + (p * (64 * 2.0 ** -24 * size + 2.0 ** -22 * (x.abs() + z.abs()) + 2.0 ** -21)).sum(0)
    w = torch.zeros((4, 20000), device="cuda")
    for i in range(2):
        evict.weigh(s.cache(), s.q, lse, s.table, s.row_starts, s.row_lengths, s.scale, w, torch.arange(4).cuda() * 20000)
    torch.cuda.synchronize()
    for r in (0, 1, 3):
        L = s.lens[r]
        off = (w[r, :L].double() - 2 * total[r]).abs() - 2 * bound[r] - (s.n_rows * 128 + 1) * 2.0 ** -23 * total[r]
        assert bool((off <= 0).all()) and not bool(w[r, L:].any()), r
    assert not bool(w[2].any())


def test_more_parts_than_the_workspace_holds_of_parts_of_rows():
    """Windows that add up in one part, each of a part of one row's heads.  (A few heads are compared: the others' lse is
    so large that they add nothing, and what they could add is below FP32's least.)"""
    from paper_2609_08450_amd import evict

    s = Setup([20000, 300], [320, 3], page=256, kv=1, heads=300, dim=64, values=False).cuda()
    assert sum(2 * n * -(-L // 256) for L, n in zip(s.lens, (320, 3))) > 49152
    picked = (0, 149, 150, 151, 299)
    lse = torch.full((s.n_rows, 300), 1e4, device="cuda")
    w = torch.zeros((2, 20000), device="cuda")
    sums = []
    for r in range(2):
        a, b, L = int(s.row_starts[r]), int(s.row_starts[r + 1]), s.lens[r]
        k, there = s.tokens("k", r, L)
        assert bool(there.all())
        hidden = torch.arange(L, device="cuda") >= s.row_lengths[a:b, None]
        total, bound = torch.zeros(L, dtype=torch.float64, device="cuda"), torch.zeros(L, dtype=torch.float64, device="cuda")
        for h in picked:
            q = s.q[a:b, h].double()
            x = s.scale * torch.matmul(q, k[0].t())
            z = torch.logsumexp(x.masked_fill(hidden, -math.inf), 1)
            lse[a:b, h] = z.float()
            z = lse[a:b, h, None].double()
            p = torch.exp(x - z).masked_fill(hidden, 0.0)
            size = s.scale * torch.matmul(q.abs(), k[0].abs().t())
            total += p.sum(0)
            bound += (p * (64 * 2.0 ** -24 * size + 2.0 ** -22 * (x.abs() + z.abs()) + 2.0 ** -21)).sum(0)
        # FP32 sums of each row's 300 heads, a rounding to a term, and of the old weight
        sums.append((total, bound + (len(q) * 300 + 1) * 2.0 ** -24 * total + 2.0 ** -24 * total))
    evict.weigh(s.cache(), s.q, lse, s.table, s.row_starts, s.row_lengths, s.scale, w, torch.tensor([0, 20000]).cuda())
    torch.cuda.synchronize()
    for r, (total, bound) in enumerate(sums):
        L = s.lens[r]
        assert bool(((w[r, :L].double() - total).abs() <= bound).all()) and not bool(w[r, L:].any()), r


def test_far_offsets():
    """Weights past 2^31 elements, and codes past 2^32 bytes."""
    from paper_2609_08450_amd import evict, paged

    s = Setup([100], [1], page=16, kv=1, heads=4, dim=64, values=False).cuda()
    n_pages = 2 ** 32 // (16 * 64) + 64
    k = torch.zeros((n_pages, 1, 16, 64), dtype=torch.uint8, device="cuda").view(E4M3)
    ks = torch.ones((n_pages, 1), device="cuda")
    at = torch.arange(7) + n_pages - 8
    used = s.table[0].long()
    k.view(torch.uint8)[at.cuda()] = s.k.view(torch.uint8)[used]
    ks[at.cuda()] = s.ks[used]
    lse = lse_of(s)
    sums = weighed(s, lse)[0][0]
    w = torch.zeros(2 ** 31 + 200, device="cuda")
    evict.weigh(paged.PagedCache.of(k, ks), s.q, lse, at.int().cuda()[None], s.row_starts, s.row_lengths, s.scale, w,
                torch.tensor([2 ** 31 + 3]).cuda())
    got = w[2 ** 31 + 3:2 ** 31 + 103].double()
    assert bool(((got - sums).abs() <= 1e-4 * sums).all()) and float(w[2 ** 31 + 103:].abs().max()) == 0.0
    assert float(w[:2 ** 31 + 3].abs().max()) == 0.0
