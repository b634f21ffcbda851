"""The chain tables -> store -> score -> Top-K -> attention as the example runs it."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_selection_of_everything_is_dense_attention():
    """While requests are no longer than K, the selected attention reads what the
    dense one reads: the outputs differ by their rounding alone (bf16: half a unit
    each, and FP32 sums and f16 weights in another order)."""
    import torch
    from examples import paged_step

    sparse, dense, _ = paged_step.run(requests=3, context=700, steps=3, K=1024, chunk=300)
    off = (sparse.float() - dense.float()).abs()
    assert bool((off <= 2.0 ** -7 * dense.float().abs() + 2.0 ** -10 * dense.float().abs().amax()).all())
    assert float(dense.float().norm()) > 0 and torch.isfinite(sparse.float()).all()


def test_the_chain_selects_what_its_scores_say():
    """A longer request: the selection is that of the scores, and the attention that
    of the selection, both against plain forms on the cache's own values."""
    import torch
    from examples import paged_step

    g = torch.Generator(device="cuda").manual_seed(3)
    server = paged_step.Server(2, 3000)
    layer = paged_step.Layer(server.n_pages, K=256)
    selector = paged_step.Selector(2600, 3000, 256)
    new = torch.tensor([2500, 60], dtype=torch.int32, device="cuda")
    server.begin(new, 2560)
    x = paged_step.activations(layer, 2560, g)
    out = paged_step.sparse_attention(server, layer, selector, **x)
    idx, val = selector.topk(selector.scores, selector.offsets[:2560], server.row_lengths)
    for row in (0, 5, 255, 256, 300, 1999, 2499, 2500, 2559):
        r, L = int(server.row_request[row]), int(server.row_lengths[row])
        P = server.page
        pages = server.table[r, :-(-L // P)].long()

        def tokens(codes, scale):
            y = codes.view(torch.uint8)[pages].view(codes.dtype).float().double() * scale[pages].double()[..., None, None]
            return y.transpose(0, 1).flatten(1, 2)[:, :L]

        ik = tokens(layer.index.k, layer.index.k_scale)
        s = (x["index_w"][row].double()[:, None] * torch.matmul(x["index_q"][row].double(), ik[0].t()).clamp(min=0)).sum(0)
        s *= layer.index_dim ** -0.5
        got = selector.scores[row, :L].double()
        assert float((got - s).abs().max()) <= 1e-5 * float(s.abs().max() + 1)
        kept = idx[row][idx[row] >= 0].long()
        assert kept.numel() == min(L, 256)
        if L > 256:
            assert float(got[kept].min()) >= float(torch.topk(got, 256).values[-1])
        k, v = tokens(layer.cache.k, layer.cache.k_scale)[:, kept], tokens(layer.cache.v, layer.cache.v_scale)[:, kept]
        q = x["q"][row].double().view(layer.kv_heads, -1, layer.dim)
        p = torch.softmax(torch.matmul(q, k.transpose(1, 2)) * layer.dim ** -0.5, -1)
        ref, mass = torch.matmul(p, v).reshape(-1, layer.dim), torch.matmul(p, v.abs()).reshape(-1, layer.dim)
        off = (out[row].double() - ref).abs()
        assert bool((off <= 2.0 ** -8 * ref.abs() + 2.0 ** -10 * mass + 2.0 ** -18 * mass.amax()).all()), row
