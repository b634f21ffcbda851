"""paged_kv_tables against its definition: every output equal."""
import pytest

from tests.paged_util import tables_oracle

pytestmark = pytest.mark.gpu

OUT = ("pool_out", "lens_out", "row_starts", "row_request", "row_lengths", "slots")


def make(n, page, width, lens, new, free, spare, seed=0):
    """A pool of `free` free pages in a ring of `spare` places more, from some place on."""
    import torch

    g = torch.Generator().manual_seed(seed)
    held = [-(-L // page) for L in lens]
    size = sum(held) + free + spare
    order = torch.randperm(size, generator=g).tolist()
    table = [[order.pop() for _ in range(h)] + [-7] * (width - h) for h in held]
    head = size - free // 2 - 1 if free else size // 2
    ring = [-9] * size
    for i in range(free):
        ring[(head + i) % size] = order.pop()
    return ring, [head, free, 5, 5], lens, new, table


def run(ring, pool, lens, new, table, page, rows, alias_pool=False, pad=0):
    import torch
    from paper_2609_08450_amd import paged

    i32 = lambda x, shape=None: torch.tensor(x, dtype=torch.int32).reshape(shape or (-1,)).cuda()  # noqa: E731
    n = len(lens)
    width = len(table[0]) if n else 1
    wide = torch.full((n, width + pad), -3, dtype=torch.int32)
    wide[:, :width] = torch.tensor(table, dtype=torch.int32).reshape(n, width)
    wide = wide.cuda()
    t = wide[:, :width]
    r, p = i32(ring), i32(pool)
    out = dict(pool_out=p if alias_pool else torch.full_like(p, -1), lens_out=i32([-1] * n), row_starts=i32([-1] * (n + 1)),
               row_request=i32([-5] * rows), row_lengths=i32([-5] * rows),
               slots=torch.full((rows,), -5, dtype=torch.int64, device="cuda"))
    paged.tables(r, p, i32(lens), i32(new), t, page, **out)
    torch.cuda.synchronize()
    assert bool((wide[:, width:] == -3).all())
    return {**{k: v.tolist() for k, v in out.items()}, "table": t.tolist(), "ring": r.tolist()}


def check(ring, pool, lens, new, table, page, rows=None, **kw):
    rows = sum(max(0, x) for x in new) if rows is None else rows
    want = tables_oracle(ring, pool, lens, new, table, page, rows)
    got = run(ring, pool, lens, new, table, page, rows, **kw)
    for k in want:
        assert got[k] == want[k], (k, [i for i, (a, b) in enumerate(zip(got[k], want[k])) if a != b][:5])


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n", [1, 3, 64, 1023, 1024, 1025, 2500, 5000])
def test_mixed_steps(n, page):
    import random

    rng = random.Random(n * page)
    lens = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, 9 * page)]) for _ in range(n)]
    new = [rng.choice([0, 1, 1, 1, page, -1, -page, -x, -x - 5, rng.randint(0, 3 * page)]) for x in lens]
    need = sum(max(0, -(-(a + b) // page) - -(-a // page)) for a, b in zip(lens, new))
    print("[case] tables mixed", n, page, flush=True)
    for free in (need, need // 2, 0):
        check(*make(n, page, 14, lens, new, free, spare=7, seed=free), page, pad=n % 3, alias_pool=free == 0)


@pytest.mark.parametrize("tokens", [1, 4096, 4097, 70001])
def test_one_prompt(tokens):
    page = 64
    check(*make(2, page, 1200, [5, 0], [-5, tokens], 1100, 3), page)


def test_more_rows_than_tokens_and_fewer():
    page = 16
    check(*make(3, page, 9, [17, 40, 0], [3, 1, 60], 20, 0), page, rows=100)
    check(*make(3, page, 9, [17, 40, 0], [3, 1, 60], 20, 0), page, rows=20)
    check(*make(3, page, 9, [17, 40, 0], [3, 1, 5000], 400, 0), page, rows=9000)  # one refused: wider than the table
    check(*make(3, page, 400, [17, 40, 0], [3, 1, 5000], 400, 0), page, rows=0)


def test_refused_requests_do_not_stop_those_that_need_no_page():
    page = 16
    # request 1 asks for more than is free; 2 needs none; 3 would fit alone but comes after
    check(*make(4, page, 40, [16, 16, 17, 16], [1, 400, 3, 1], 3, 0), page)


def test_released_pages_serve_the_same_step():
    page = 32
    check(*make(2, page, 9, [0, 200], [150, -200], 0, 0), page)


@pytest.mark.parametrize("rows", [50, 9000])
@pytest.mark.parametrize("more", [[], [1] * 2000])
def test_rows_past_32_bits(rows, more):
    """Refused requests that ask for more rows than 32 bits count, before one that is served."""
    page, most = 16, 2 ** 31 - 1
    lens, new = [0, 0, 20, 0] + [0] * len(more), [most, 2 ** 30, 5, 1] + more
    print("[case] tables, rows past 32 bits", rows, len(more), flush=True)
    got = run(*make(len(lens), page, 9, lens, new, 10, 0), page, rows)
    assert got["row_starts"] == [0] + [most] * len(lens)
    assert got["row_request"] == [0] * rows and got["row_lengths"] == [0] * rows and got["slots"] == [-1] * rows
    served = min(10, 1 + len(more))  # pages go to the requests of one token, in order
    assert got["lens_out"] == [0, 0, 25] + [1] * served + [0] * (1 + len(more) - served)
    assert got["pool_out"][1:] == [10 - served, 2 + 1 + len(more) - served, 0]


def test_no_requests():
    check([3, 1, 2], [1, 2, 0, 0], [], [], [], 16, rows=4)
    check([3, 1, 2], [1, 2, 0, 0], [], [], [], 16, rows=5000)


def test_any_pool_state_stays_inside():
    """A state that no call leaves: places and counts outside the ring."""
    page = 16
    ring, pool, lens, new, table = make(3, page, 9, [17, 40, 0], [30, -40, 60], 20, 0)
    for state in ([-1, 20, 0, 0], [10 ** 9, 10 ** 9, 0, 0], [5, -20, 0, 0]):
        got = run(ring, state, lens, new, table, page, 90)
        assert len(got["slots"]) == 90


def test_steps_in_a_graph():
    """Two steps, lengths back and forth between two buffers, captured and replayed
    with eager work between the replays."""
    import torch
    from paper_2609_08450_amd import paged

    n, page, width, rows = 5, 16, 64, 5
    i32 = dict(dtype=torch.int32, device="cuda")
    ring, pool = torch.randperm(400).int().cuda(), torch.tensor([0, 400, 0, 0], **i32)
    table = torch.full((n, width), -1, **i32)
    a, b = torch.zeros(n, **i32), torch.zeros(n, **i32)
    new = torch.ones(n, **i32)
    o = dict(row_starts=torch.empty(n + 1, **i32), row_request=torch.empty(rows, **i32),
             row_lengths=torch.empty(rows, **i32), slots=torch.empty(rows, dtype=torch.int64, device="cuda"))

    def two():
        paged.tables(ring, pool, a, new, table, page, pool_out=pool, lens_out=b, **o)
        paged.tables(ring, pool, b, new, table, page, pool_out=pool, lens_out=a, **o)

    two()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two()
    for step in range(2, 40):
        graph.replay()
        torch.cuda.synchronize()
        assert a.tolist() == [2 * step] * n
        pages = -(-2 * step // page)
        used = table[:, :pages].reshape(-1).tolist()
        assert len(set(used)) == len(used) and pool[1].item() == 400 - len(used) and min(used) >= 0
        want = table[:, (2 * step - 1) // page].long() * page + (2 * step - 1) % page
        assert torch.equal(o["slots"], want) and o["row_lengths"].tolist() == [2 * step] * n
