"""Paged calls on a stream that is not the current one."""
import pytest
import torch

from tests.paged_util import Setup, assert_attention, attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("selected", [False, True])
def test_an_output_that_a_call_makes_belongs_to_its_stream(selected):
    """The current stream still has to fill a tensor that is freed: a call on another
    stream does not get its memory."""
    from paper_2609_08450_amd import paged

    s = Setup([700, 300], [1, 1], page=32, kv=2, heads=8, dim=128).cuda()
    idx = torch.arange(500, dtype=torch.int32, device="cuda").repeat(2, 1)
    ref = attention(s, idx if selected else None)
    cache, side = s.cache(), torch.cuda.Stream()
    ws = cache.alloc_workspace(2, 2, 8)
    filler = torch.ones(1 << 26, device="cuda")
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for _ in range(50):
            filler.mul_(1.0)  # the current stream is busy meanwhile
        freed = torch.empty_like(s.q)
        freed.fill_(7.0)
        where = freed.data_ptr()
        del freed
        if selected:
            out = paged.attend_selected(cache, s.q, idx, s.table, s.row_request, s.row_lengths, s.scale, workspace=ws,
                                        stream=stream)
        else:
            out = paged.attend(cache, s.q, s.table, s.row_starts, s.row_lengths, s.scale, workspace=ws, stream=stream)
        assert out.data_ptr() != where
        torch.cuda.synchronize()
        assert_attention(out, None, ref, "output of another stream")


def test_the_default_streams_handle():
    """A program may hand over the number of the stream that is current, 0 for the default one."""
    from paper_2609_08450_amd import paged

    s = Setup([700, 300], [1, 1], page=32, kv=2, heads=8, dim=128).cuda()
    ref, cache = attention(s), s.cache()
    assert torch.cuda.current_stream().cuda_stream == 0
    for _ in range(2):  # with the workspace's first call, and after it
        out = paged.attend(cache, s.q, s.table, s.row_starts, s.row_lengths, s.scale, stream=0)
        torch.cuda.synchronize()
        assert_attention(out, None, ref, "stream 0")
    assert torch.cuda.current_stream().cuda_stream == 0
