"""The workspace that a PagedCache keeps for its attention calls."""
import gc
import weakref

import pytest
import torch

from tests.paged_util import Setup, assert_attention, attention


def bare(paged, monkeypatch, sizes):
    """A cache on the CPU whose calls need sizes[n_rows] bytes."""
    monkeypatch.setattr(paged.PagedCache, "workspace_size", lambda self, rows, requests, heads: sizes[rows])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    cache = paged.PagedCache.__new__(paged.PagedCache)
    cache.k, cache.workspace, cache._replaced = torch.zeros(1), None, []
    return cache


def test_a_replaced_workspace_stays(monkeypatch):
    """A captured graph, or a call on another stream, may still use it."""
    from paper_2609_08450_amd import paged

    cache = bare(paged, monkeypatch, {1: 9000, 2: 40 << 20, 3: 20000})
    at, size = cache._space(None, 1, 1, 8, None)
    assert at == cache.workspace.data_ptr() and size >= 9000
    first = weakref.ref(cache.workspace.untyped_storage())
    at = cache._space(None, 2, 1, 8, None)[0]
    assert cache._space(None, 3, 1, 8, None)[0] == at == cache.workspace.data_ptr()
    gc.collect()
    assert first() is not None


def test_a_workspace_that_grows_slowly_is_replaced_seldom(monkeypatch):
    """One row more with each call: what is kept stays a small multiple of what is needed."""
    from paper_2609_08450_amd import paged

    sizes = {n: (60 << 20) + 20 * n for n in range(1, 200001)}
    cache = bare(paged, monkeypatch, sizes)
    for n in range(1, 200001, 50):
        assert cache._space(None, n, 1, 8, None)[1] >= sizes[n]
    assert cache.workspace.numel() + sum(x.numel() for x in cache._replaced) <= 2 * sizes[1]


@pytest.mark.gpu
def test_a_graph_outlives_its_caches_workspace():
    """Captured with the cache's workspace; then a call that needs a larger one, and
    tensors filled over whatever memory is free; then the replays."""
    from paper_2609_08450_amd import paged

    s = Setup([9000, 200], [1, 1], page=32, kv=2, heads=8, dim=128).cuda()
    big = Setup([600, 500], [400, 100], page=32, kv=2, heads=8, dim=128).cuda()
    cache, out = s.cache(), torch.empty_like(s.q)
    torch.cuda.synchronize()
    paged.attend(cache, s.q, s.table, s.row_starts, s.row_lengths, s.scale, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        paged.attend(cache, s.q, s.table, s.row_starts, s.row_lengths, s.scale, out=out)
    first = cache.workspace
    where, size = first.data_ptr(), first.numel()
    del first
    ref = attention(s)
    for i in range(3):
        paged.attend(cache, big.q, s.table, big.row_starts, big.row_lengths.clamp(max=200), s.scale)
        assert cache.workspace.data_ptr() != where and cache.workspace.numel() > size
        filled = [torch.full((size,), 0x7B, dtype=torch.uint8, device="cuda") for _ in range(4)]
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((x == 0x7B).all()) for x in filled)
        assert_attention(out, None, ref, f"replay {i}")
        del filled


@pytest.mark.gpu
def test_no_workspace_is_made_under_capture():
    """It would be zeroed by the replays alone, and be the graph's memory: calls before
    the first replay would find tickets that are not zero."""
    from paper_2609_08450_amd import paged

    s = Setup([9000, 200], [1, 1], page=32, kv=2, heads=8, dim=128).cuda()
    cache, out, x = s.cache(), torch.empty_like(s.q), torch.zeros(8, device="cuda")
    args = (s.table, s.row_starts, s.row_lengths, s.scale)
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):  # the capturing stream is the current one, or given
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            x.add_(1.0)
            with pytest.raises(paged.PagedError, match="capture"):
                paged.attend(cache, s.q, *args, out=out, stream=stream)
            x.add_(1.0)
        assert cache.workspace is None
    graph.replay()
    ref = attention(s)
    paged.attend(cache, s.q, *args, out=out)
    torch.cuda.synchronize()
    assert_attention(out, None, ref, "after a refused capture")
    # a larger one neither; what fits the one that is there is captured
    big = Setup([600], [500], page=32, kv=2, heads=8, dim=128).cuda()
    had, graph = cache.workspace, torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(paged.PagedError, match="capture"):
            paged.attend(cache, big.q, s.table[:1], big.row_starts, big.row_lengths, s.scale)
        paged.attend(cache, s.q, *args, out=out)
    assert cache.workspace is had
    for i in range(3):
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert_attention(out, None, ref, f"replay {i}")
