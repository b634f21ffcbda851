"""paged_kv_attend and paged_kv_attend_selected against 64-bit attention."""
import pytest
import torch

from tests.paged_util import Setup, assert_attention, attention

pytestmark = pytest.mark.gpu

CODE = [torch.float8_e4m3fn, torch.int8]
ACT = [torch.bfloat16, torch.float16]


def run(s, picked=None, cache=None, **kw):
    from paper_2609_08450_amd import paged

    c = cache or s.cache()
    out = torch.full((s.n_rows, s.heads, s.dim), 7.0, dtype=s.act, device="cuda")
    lse = torch.full((s.n_rows, s.heads), 7.0, device="cuda")
    if picked is None:
        got = paged.attend(c, s.q, s.table, s.row_starts, s.row_lengths, s.scale, out=out, lse=lse, **kw)
    else:
        got = paged.attend_selected(c, s.q, picked, s.table, s.row_request, s.row_lengths, s.scale, out=out, lse=lse, **kw)
    assert got is out
    torch.cuda.synchronize()
    return out, lse


def check(s, picked=None, where="", **kw):
    print("[case]", where, "rows", s.n_rows, "heads", s.heads, s.kv, "dim", s.dim, "page", s.page, s.k.dtype, s.act,
          flush=True)
    s.cuda()
    out, lse = run(s, picked, **kw)
    assert_attention(out, lse, attention(s, picked), where)
    return out, lse


def selection(s, K, seed=0, junk=True):
    """K tokens of each row, unordered, some absent: -1, past the row's end, and huge."""
    g = torch.Generator().manual_seed(seed)
    idx = torch.full((s.n_rows, K), -1, dtype=torch.int32)
    for i, L in enumerate(s.row_lengths.tolist()):
        p = torch.randperm(max(L, 1), generator=g)[:K][:max(L, 0)].int()
        idx[i, :len(p)] = p
        if junk and i % 3 == 1:
            idx[i] = idx[i, torch.randperm(K, generator=g)]
            bad = torch.randint(0, K, (max(1, K // 5),), generator=g)
            idx[i, bad] = torch.tensor([-1, L, L + 1000, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).repeat(K)[:len(bad)]
    return idx.cuda()


# Single tokens: one row to a request.

@pytest.mark.parametrize("code", CODE, ids=str)
@pytest.mark.parametrize("act", ACT, ids=str)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens(code, act, dim, page):
    lens = [1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 1000, 3001, 0]
    check(Setup(lens, [1] * len(lens), page=page, dim=dim, code=code, act=act), where="single")


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (15, 5), (16, 1), (17, 1), (32, 2), (33, 1), (64, 1), (128, 2), (6, 6)])
def test_head_layouts(heads, kv):
    lens = [700, 33, 1]
    for act in ACT:
        check(Setup(lens, [1, 1, 1], heads=heads, kv=kv, dim=64, act=act, page=32), where="heads")
        check(Setup(lens, [9, 2, 1], heads=heads, kv=kv, dim=128, act=act, page=32), where="heads of a prompt")


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_more_heads_than_a_group_has_columns(dim):
    """A row's heads on one cache head are cut into parts, the last one not full."""
    for lens, rows in (([700, 33], [1, 1]), ([700, 33], [9, 2]), ([20000], [5])):
        check(Setup(lens, rows, heads=300, kv=1, dim=dim, page=32), where="many heads")


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_one_long_row(page):
    """One row over the whole card: many workgroups join their parts."""
    check(Setup([60001], [1], page=page, kv=1, heads=5, dim=128), where="long")


def test_many_rows():
    lens = [(7 * i * i) % 611 for i in range(1500)]
    check(Setup(lens, [1] * 1500, kv=1, heads=2, dim=64), where="many")


# Prompts: many rows to a request.

@pytest.mark.parametrize("code", CODE, ids=str)
@pytest.mark.parametrize("act", ACT, ids=str)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 128])
def test_prompts(code, act, dim, page):
    check(Setup([300, 64, 1, 700, 65, 0, 129], [300, 64, 1, 70, 2, 0, 5], page=page, dim=dim, code=code, act=act),
          where="prompts")


@pytest.mark.parametrize("rows", [2, 3, 31, 32, 33, 500])
def test_chunks_of_a_long_prompt(rows):
    check(Setup([9000], [rows], page=64, kv=2, heads=6, dim=128), where="chunk")


def test_prompts_beside_single_tokens():
    lens = [2000, 5, 900, 33, 70, 4000]
    check(Setup(lens, [1, 1, 200, 1, 30, 1], page=32, kv=2, heads=8, dim=128), where="mixed")


# Rows that see nothing, or less than their request.

@pytest.mark.parametrize("prompt", [False, True])
def test_rows_that_see_nothing(prompt):
    lens = [40, 100, 7, 64]
    rows = [1, 1, 1, 1] if not prompt else [3, 2, 5, 4]
    n = sum(rows)
    seen = [0, 55, -5, 64] if not prompt else [0, 3, 40, 0, 0, 7, 0, 1, -9, 2, 64, 0, 1, 63]
    s = Setup(lens, rows, dim=64, seen=seen[:n])
    out, lse = check(s, where="empty rows")
    for i, L in enumerate(seen):
        assert L > 0 or (bool((out[i] == 0).all()) and bool((lse[i] == -torch.inf).all()))


@pytest.mark.parametrize("prompt", [False, True])
def test_rows_of_no_request(prompt):
    """row_starts ends before the rows do."""
    s = Setup([50, 60], [1, 1] if not prompt else [4, 5], dim=128)
    extra = 2 if prompt else 0
    s.q = torch.cat([s.q, s.q[:1].repeat(extra, 1, 1)])
    s.row_lengths = torch.cat([s.row_lengths, torch.full((extra,), 9, dtype=torch.int32)])
    s.n_rows += extra
    if not prompt:
        s.row_starts[2] = 1
        s.row_request = s.row_request[:1]
    out, lse = check(s, where="no request")
    assert bool((out[int(s.row_starts[2]):] == 0).all()) and bool((lse[int(s.row_starts[2]):] == -torch.inf).all())


@pytest.mark.parametrize("before,rows,after", [(1, [1, 1], 0), (2, [1, 0, 1], 2), (3, [4, 5], 0), (3, [4, 0, 5], 2),
                                               (700, [40, 3], 300)])
def test_rows_before_the_first_request(before, rows, after):
    """row_starts begins after the rows do: single rows and prompts."""
    s = Setup([50 + i for i in range(len(rows))], rows, dim=64)
    n = s.n_rows
    s.q = torch.cat([s.q[:1].repeat(before, 1, 1), s.q, s.q[:1].repeat(after, 1, 1)])
    s.row_lengths = torch.cat([torch.full((before,), 9, dtype=torch.int32), s.row_lengths,
                               torch.full((after,), 9, dtype=torch.int32)])
    s.row_request = torch.cat([torch.full((before,), -1, dtype=torch.int32), s.row_request])
    s.row_starts += before
    s.n_rows += before + after
    out, lse = check(s, where="rows before")
    for part in (slice(0, before), slice(before + n, None)):
        assert bool((out[part] == 0).all()) and bool((lse[part] == -torch.inf).all())


def test_rows_of_no_requests_at_all():
    from paper_2609_08450_amd import paged

    s = Setup([50], [5], dim=64).cuda()
    for start in (0, 2, 5, 9):
        out, lse = torch.full_like(s.q, 7.0), torch.full((5, 8), 7.0, device="cuda")
        paged.attend(s.cache(), s.q, s.table[:0], torch.tensor([start], dtype=torch.int32).cuda(), s.row_lengths, s.scale,
                     out=out, lse=lse)
        assert bool((out == 0).all()) and bool((lse == -torch.inf).all())


@pytest.mark.parametrize("prompt", [False, True])
def test_pages_outside_the_cache_are_absent(prompt):
    s = Setup([200, 90, 33], [1, 1, 1] if not prompt else [150, 20, 3], page=16, dim=64)
    s.table[0, 3], s.table[0, 7], s.table[1, 0], s.table[2, :] = -1, s.n_pages, 2 ** 31 - 1, -5
    check(s, where="absent pages")


@pytest.mark.parametrize("prompt", [False, True])
def test_lengths_end_with_the_table(prompt):
    s = Setup([64, 32], [1, 1] if not prompt else [2, 3], page=16, dim=64)
    s.row_lengths[:] = 10 ** 6
    s.table[1, 2:] = -1
    check(s, where="table's end")


def test_lengths_need_not_rise():
    g = torch.Generator().manual_seed(4)
    seen = torch.randint(0, 400, (300,), generator=g).tolist()
    check(Setup([400], [300], page=32, kv=1, heads=4, dim=128, seen=seen), where="any lengths")


def test_scales_far_apart():
    """A page's scale does not cost the others their precision."""
    for prompt in (False, True):
        s = Setup([500, 300], [1, 1] if not prompt else [40, 9], page=16, dim=128, act=torch.float16, q_scale=1.0)
        s.vs[:] = 2.0 ** torch.randint(-30, 0, s.vs.shape, generator=torch.Generator().manual_seed(1)).float() / 448
        check(s, where="scales")
        s = Setup([500], [1], page=16, dim=128, act=torch.float16, q_scale=1.0)
        s.vs[:] = 0.0
        check(s, where="zero scales")


def test_peaked_and_large_scores():
    for prompt in (False, True):
        check(Setup([3000], [1] if not prompt else [64], page=64, dim=128, q_scale=40.0, act=torch.float16),
              where="peaked")


def far_scales(lens, rows, ratio, where, code, act, dim=128, heads=8, seen=None):
    """Pages `where` of each request have values 2^ratio times as large as the others,
    and keys that queries of one sign do not look at (a weight of about e^-80) while
    those of the other sign look at nothing else."""
    s = Setup(lens, rows, page=16, kv=2, heads=heads, dim=dim, code=code, act=act, seen=seen)
    g = torch.Generator().manual_seed(ratio)
    shift = torch.full((s.n_pages, 1, 1, 1), 0.5)
    s.vs[:] = 2.0 ** -6
    for t in s.table.tolist():
        for j in where:
            if j < len(t) and t[j] >= 0:
                shift[t[j]] = -0.5
                s.vs[t[j]] = 2.0 ** (ratio - 6)
    k = 0.05 * torch.randn(s.k.shape, generator=g) + shift
    s.ks[:] = 1 / 64
    s.k = (k * 64).round().to(code) if code is torch.int8 else (k * 64).to(code)
    sign = 1 - 2 * torch.randint(0, 2, (s.n_rows, heads, 1), generator=g)
    sign[::3] = 1  # most look at the others
    s.q = ((7 * sign + 0.3 * torch.randn(s.q.shape, generator=g)) * (128 / dim) ** 0.5).to(act)
    return s


def check_far(s, picked=None):
    """Each row and head against its own mass.  Weights are rounded to f16 and follow
    scores that FP32 holds (a part in 2^24 for each of the products); a weight below f16's
    normal ones is off by 2^-25 of a unit that is at most 2^-6 of the row's largest product of weight and
    scale, which is at most the sum of them (the mass of values of 1)."""
    s.cuda()
    out, lse = run(s, picked)
    ref, ref_lse, mass = attention(s, picked)
    one = Setup.__new__(Setup)
    vars(one).update(vars(s), v=torch.ones_like(s.v.float()).to(s.v.dtype))
    weighed = attention(one, picked)[0]
    tokens = int(s.row_lengths.max()) if picked is None else picked.shape[1]
    unit, least = (2.0 ** -8, 2.0 ** -133) if s.act is torch.bfloat16 else (2.0 ** -11, 2.0 ** -25)
    empty = ref_lse == -torch.inf
    score = s.dim * 2.0 ** -24 * float(ref_lse[~empty].abs().max())
    tol = unit * ref.abs() + (2.0 ** -10 + 2 * score) * mass + tokens * 448 * 2.0 ** -31 * weighed + least
    off = (out.double() - ref).abs()
    over = ref.abs() + tol > torch.finfo(s.act).max  # past f16's largest
    bad = (off > tol) & ~over
    assert not bool(bad.any()), (f"{int(bad.sum())} of {bad.numel()} out of bounds, first at {bad.nonzero()[0].tolist()}: "
                                 f"{float(out[bad][0])} for {float(ref[bad][0])}")
    assert bool((lse[empty] == -torch.inf).all()) and bool((out[empty] == 0).all())
    assert bool(((lse.double() - ref_lse)[~empty].abs() <= 2.0 ** -15 * (1 + ref_lse[~empty].abs())).all())


@pytest.mark.parametrize("code", CODE, ids=str)
@pytest.mark.parametrize("act", ACT, ids=str)
@pytest.mark.parametrize("ratio", [-40, 8, 16, 22, 30, 50])
@pytest.mark.parametrize("lens,rows,where", [([600, 50], [1, 1], [0]), ([600, 50], [1, 1], [3, 20]), ([600], [1], [36]),
                                             ([600, 90], [60, 5], [0, 1]), ([600, 90], [600, 90], [2, 17, 30])])
def test_pages_that_weigh_nothing_cost_no_precision(code, act, ratio, lens, rows, where):
    """However large their values, and whether other rows look at them or see them."""
    print("[case] far scales", lens, rows, where, ratio, code, act, flush=True)
    s = far_scales(lens, rows, ratio, where, code, act)
    idx = selection(s, 300)
    check_far(s)
    check_far(s, idx)


@pytest.mark.parametrize("dim,heads", [(64, 8), (256, 8), (128, 40), (64, 66)])
@pytest.mark.parametrize("rows", [[1, 1], [200, 30]])
def test_far_scales_of_other_heads(dim, heads, rows):
    s = far_scales([600, 50], rows, 30, [0, 9], torch.float8_e4m3fn, torch.bfloat16, dim=dim, heads=heads)
    idx = selection(s, 300)
    check_far(s)
    check_far(s, idx)


def test_rows_that_do_not_see_the_large_values():
    """In prompts: pages that only later rows of the group see."""
    seen = [100, 100, 600, 600, 90, 33, 17, 600] * 5
    s = far_scales([600], [40], 40, [8, 9, 30], torch.float8_e4m3fn, torch.float16, seen=seen)
    check_far(s)


def test_zero_scales_beside_others():
    """Pages of scale 0 (and keys' scales of 0) hold weight but no values."""
    for rows in ([1, 1], [60, 20]):
        s = far_scales([600, 50], rows, 0, [0, 1, 9], torch.float8_e4m3fn, torch.bfloat16)
        g = torch.Generator().manual_seed(5)
        s.vs[torch.rand(s.vs.shape, generator=g) < 0.4] = 0.0
        s.ks[torch.rand(s.ks.shape, generator=g) < 0.2] = 0.0
        idx = selection(s, 300)
        check_far(s)
        check_far(s, idx)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens,rows", [([40, 50], [1, 1]), ([30000, 50], [1, 1]), ([300, 50], [40, 1]), ([9000, 50], [100, 1])])
def test_queries_that_are_not_finite_show(lens, rows, bad):
    """A head's NaN is its result, in one part or joined from many, and no other head's."""
    s = Setup(lens, rows, page=32, kv=2, heads=8, dim=128)
    s.q[1, 3], s.q[0, 6, 5] = bad, bad
    s.cuda()
    hit = torch.zeros((s.n_rows, 8), dtype=torch.bool, device="cuda")
    hit[1, 3] = hit[0, 6] = True
    finite = s.q.clone()
    finite[hit] = 1.0
    idx = torch.arange(3000, dtype=torch.int32, device="cuda").repeat(s.n_rows, 1)
    for picked in (None, idx):
        out, lse = run(s, picked)
        assert bool(torch.isnan(out[hit]).all()) and bool(torch.isnan(lse[hit]).all())
        t = Setup.__new__(Setup)
        vars(t).update(vars(s), q=finite)
        assert torch.equal(out[~hit], run(t, picked)[0][~hit])


# Layouts.

@pytest.mark.parametrize("prompt", [False, True])
def test_strided_queries_tables_and_pages(prompt):
    s = Setup([333, 70], [1, 1] if not prompt else [33, 7], page=32, kv=2, heads=8, dim=128).cuda()
    ref = attention(s)
    wide = torch.full((s.n_rows, 14, 136), float("nan"), dtype=s.act, device="cuda")
    wide[:, 2:10, :128] = s.q
    s.q = wide[:, 2:10, :128]
    t = torch.full((2, s.table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    t[:, :s.table.shape[1]] = s.table
    s.table = t[:, :s.table.shape[1]]
    for a, b in (("k", "ks"), ("v", "vs")):
        x = getattr(s, a)
        w = torch.full((x.shape[0], 3, *x.shape[1:]), 0x7F, dtype=torch.uint8, device="cuda")
        w[:, 1] = x.view(torch.uint8)
        setattr(s, a, w.view(x.dtype)[:, 1])
        sc = torch.full((x.shape[0], 3, x.shape[1]), float("nan"), device="cuda")
        sc[:, 1] = getattr(s, b)
        setattr(s, b, sc[:, 1])
    out, lse = run(s)
    assert_attention(out, lse, ref, "strides")


@pytest.mark.parametrize("prompt", [False, True])
def test_a_cache_past_32_bit_offsets(prompt):
    """Pages whose bytes lie past 2^32."""
    from paper_2609_08450_amd import paged

    s = Setup([300, 77], [1, 1] if not prompt else [40, 3], page=64, kv=2, heads=8, dim=128).cuda()
    far = 2 ** 32 // (2 * 64 * 128) + 12345
    cache = paged.PagedCache(far + s.n_pages, 64, 2, 128)
    cache.k[far:], cache.v[far:] = s.k, s.v
    cache.k_scale[far:], cache.v_scale[far:] = s.ks, s.vs
    ref = attention(s)
    idx = selection(s, 100, junk=False)
    ref_picked = attention(s, idx)
    s.table = torch.where(s.table >= 0, s.table + far, s.table)
    assert_attention(*run(s, cache=cache), ref, "far pages")
    assert_attention(*run(s, idx, cache=cache), ref_picked, "far pages, selected")


# Selected tokens.

@pytest.mark.parametrize("code", CODE, ids=str)
@pytest.mark.parametrize("act", ACT, ids=str)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("K", [1, 31, 128, 200, 1025, 2500])
def test_selected(code, act, dim, K):
    lens = [1, 40, 900, 3000, 17, 0, 2000]
    s = Setup(lens, [1, 2, 3, 1, 4, 1, 2], page=32, kv=2, heads=8, dim=dim, code=code, act=act)
    check(s, selection(s, K), where=f"selected {K}")


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (17, 1), (33, 1), (128, 2), (6, 6)])
def test_selected_head_layouts(heads, kv):
    s = Setup([500, 60], [3, 2], page=16, kv=kv, heads=heads, dim=64)
    check(s, selection(s, 300), where="selected heads")


def test_selected_many_rows():
    s = Setup([4000, 100], [1100, 30], page=64, kv=1, heads=16, dim=128)
    check(s, selection(s, 160), where="selected, many rows")


def test_selected_reads_what_is_selected_alone():
    """Tokens that no row selects are NaN."""
    s = Setup([600], [4], page=16, kv=2, heads=4, dim=64)
    idx = selection(s, 64, junk=False)
    keep = torch.zeros(600, dtype=torch.bool)
    keep[idx.cpu().long().reshape(-1)] = True
    for x in (s.k, s.v):
        for t in (~keep).nonzero()[:, 0].tolist():
            x.view(torch.uint8)[s.table[0, t // 16], :, t % 16] = 0x7F
    check(s, idx, where="selected alone")


def test_selected_twice_counts_twice():
    s = Setup([50], [1], page=16, kv=1, heads=4, dim=64)
    idx = torch.tensor([[3, 3, 3, 9, 48, -1, 9]], dtype=torch.int32).cuda()
    check(s, idx, where="twice")


def test_selected_rows_of_no_request():
    s = Setup([50, 60], [2, 2], page=16, kv=1, heads=4, dim=64)
    idx = selection(s, 20, junk=False)
    s.row_request[1], s.row_request[2] = -1, 2
    s.table[1, 1] = -1
    out, lse = check(s, idx, where="no request")
    assert bool((out[1:3] == 0).all()) and bool((lse[1:3] == -torch.inf).all())


# Calls as a program makes them.

def test_workspace_is_ready_for_the_next_call():
    """Calls of every shape in turn on one workspace, twice: tickets are back at zero."""
    shapes = [dict(lens=[9000], rows=[1]), dict(lens=[400, 900], rows=[200, 100]), dict(lens=[50] * 70, rows=[1] * 70),
              dict(lens=[30000], rows=[3]), dict(lens=[20], rows=[1])]
    made = [Setup(page=32, kv=2, heads=8, dim=128, seed=i, **kw).cuda() for i, kw in enumerate(shapes)]
    refs = [attention(s) for s in made]
    lists = [selection(s, 700, junk=False) for s in made]
    picked = [attention(s, i) for s, i in zip(made, lists)]
    space = None
    for s in made:
        ws = s.cache().alloc_workspace(s.n_rows, len(s.lens), s.heads)
        space = ws if space is None or ws.numel() > space.numel() else space
    for _ in range(2):
        for s, ref, idx, pick in zip(made, refs, lists, picked):
            assert_attention(*run(s, workspace=space), ref, "shared workspace")
            assert_attention(*run(s, idx, workspace=space), pick, "shared workspace, selected")
    torch.cuda.synchronize()
    assert int(space[:8192].max()) == 0


def test_two_streams():
    made = [Setup([5000 + i, 70], [1, 1] if i else [40, 1], page=32, kv=2, heads=8, dim=128, seed=i).cuda()
            for i in range(2)]
    refs = [attention(s) for s in made]
    caches = [s.cache() for s in made]
    streams = [torch.cuda.Stream() for _ in made]
    outs = []
    torch.cuda.synchronize()
    from paper_2609_08450_amd import paged

    spaces = [c.alloc_workspace(s.n_rows, 2, 8) for s, c in zip(made, caches)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, c, st, ws in zip(made, caches, streams, spaces):
            out, lse = torch.empty_like(s.q), torch.empty((s.n_rows, s.heads), device="cuda")
            paged.attend(c, s.q, s.table, s.row_starts, s.row_lengths, s.scale, out=out, lse=lse, workspace=ws, stream=st)
            outs.append((out, lse))
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(outs):
        assert_attention(out, lse, refs[i % 2], "streams")


def test_first_call_on_a_stream_of_its_own():
    """The cache's own workspace is made ready on the stream that uses it."""
    from paper_2609_08450_amd import paged

    s = Setup([9000], [1], page=32, kv=1, heads=8, dim=128).cuda()
    ref, other = attention(s), torch.cuda.Stream()
    filler = torch.ones(1 << 26, device="cuda")
    torch.cuda.synchronize()
    for handle in (other, other.cuda_stream):
        for _ in range(4):
            filler.mul_(1.0)  # the current stream is busy meanwhile
        out, lse = torch.empty_like(s.q), torch.empty((1, 8), device="cuda")
        other.wait_stream(torch.cuda.current_stream())
        paged.attend(s.cache(), s.q, s.table, s.row_starts, s.row_lengths, s.scale, out=out, lse=lse, stream=handle)
        torch.cuda.synchronize()
        assert_attention(out, lse, ref, "own stream")


@pytest.mark.parametrize("prompt", [False, True])
def test_graph(prompt):
    """Captured once, replayed with eager calls between, each replay on other inputs."""
    s = Setup([3000, 200], [1, 1] if not prompt else [100, 1], page=32, kv=2, heads=8, dim=128).cuda()
    cache = s.cache()
    idx = selection(s, 300, junk=False)
    run(s, cache=cache)
    run(s, idx, cache=cache)
    from paper_2609_08450_amd import paged

    out, out2 = torch.empty_like(s.q), torch.empty_like(s.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        paged.attend(cache, s.q, s.table, s.row_starts, s.row_lengths, s.scale, out=out)
        paged.attend_selected(cache, s.q, idx, s.table, s.row_request, s.row_lengths, s.scale, out=out2)
    for i in range(5):
        s.q.copy_(torch.randn(s.q.shape, generator=torch.Generator().manual_seed(i)).to(s.act))
        s.row_lengths[0] = 2000 + 100 * i
        graph.replay()
        torch.cuda.synchronize()
        ref, pick = attention(s), attention(s, idx)
        assert_attention(out, None, ref, f"replay {i}")
        assert_attention(out2, None, pick, f"replay {i}, selected")
        assert torch.equal(out, run(s, cache=cache)[0])


def test_calls_repeat_to_the_bit():
    """Parts are joined in order, whoever arrives last."""
    for s in (Setup([20000], [1], page=64, kv=1, heads=8, dim=128), Setup([6000], [300], page=64, kv=1, heads=8, dim=128)):
        s.cuda()
        first = run(s)
        idx = selection(s, 2000, junk=False)
        second = run(s, idx)
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(first, run(s)))
            assert all(torch.equal(a, b) for a, b in zip(second, run(s, idx)))


def test_refusals():
    from paper_2609_08450_amd import paged

    s = Setup([50, 60], [1, 1], dim=64).cuda()
    c = s.cache()
    args = [c, s.q, s.table, s.row_starts, s.row_lengths, s.scale]
    for at, bad in ((1, s.q.float()), (1, s.q[..., :32]), (1, s.q[:, :3]), (1, s.q.transpose(0, 2)), (2, s.table.long()),
                    (2, s.table[:1]), (3, s.row_starts[:2]), (3, s.row_starts.long()), (4, s.row_lengths[:1])):
        a = list(args)
        a[at] = bad
        with pytest.raises(paged.PagedError):
            paged.attend(*a)
    with pytest.raises(paged.PagedError, match="workspace too small"):
        paged.attend(*args, workspace=torch.zeros(4096, dtype=torch.uint8, device="cuda"))
    with pytest.raises(paged.PagedError):
        paged.attend(*args, out=torch.empty((2, 8, 64), device="cuda"))
    with pytest.raises(paged.PagedError):
        paged.attend_selected(c, s.q, selection(s, 5).long(), s.table, s.row_request, s.row_lengths, s.scale)
    with pytest.raises(paged.PagedError):
        paged.attend(paged.PagedCache(2, 16, 2, 64, values=False), *args[1:])
    assert paged.attend(c, s.q[:0], s.table, s.row_starts, s.row_lengths[:0], s.scale).shape == (0, 8, 64)
