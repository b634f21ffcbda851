"""Rotary positions against their definition in 64 bits."""
import math

import pytest
import torch

from tests.serve_util import assert_rotated, rotated

TYPES = [torch.bfloat16, torch.float16, torch.float32]
gpu = pytest.mark.gpu


def unsigned(rope):
    return [t % 2 ** 64 for t in rope.turns.tolist()]


def check(rope, positions, q, k=None, where="", **how):
    """rotate() to new tensors against the definition."""
    from paper_2609_08450_amd import rotary

    transposed = how.get("transposed", False)
    got = rotary.rotate(rope, positions, q, k, **how)
    torch.cuda.synchronize()
    il = rope.layout == "interleaved"
    for x, y in ((q, got if k is None else got[0]),) + (() if k is None else ((k, got[1]),)):
        ref = rotated(unsigned(rope), rope.magnitude, positions.tolist(), x.cpu(), rope.start, il, transposed)
        assert_rotated(y, ref, rope.magnitude, where)
    return got


# dim, rot, start: whole 16-byte pieces, pieces of 4, 2 and 1 elements, parts in front, behind and inside
SHAPES = [(64, 64, 0), (128, 128, 0), (256, 64, 192), (80, 40, 0), (96, 24, 72), (96, 48, 20), (33, 6, 5), (2, 2, 0),
          (7, 2, 1), (130, 130, 0), (1024, 1024, 0)]


@gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("act", TYPES, ids=str)
@pytest.mark.parametrize("dim,rot,start", SHAPES)
def test_shapes(dim, rot, start, act, layout):
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(dim + rot)
    rope = rotary.Rotary(rot, layout=layout, start=start)
    q, k = (torch.randn((5, h, dim), generator=g).to(act).cuda() for h in (6, 1))
    positions = torch.tensor([0, 1, 4095, 70001, 1], dtype=torch.int32).cuda()
    check(rope, positions, q, k)
    check(rope, positions, q, transposed=True)


@gpu
@pytest.mark.parametrize("rows,heads,kv", [(1, 1, 0), (1, 64, 8), (3, 17, 5), (600, 2, 1), (2500, 3, 0)])
def test_sizes(rows, heads, kv):
    """From a single head to several rows of a workgroup, and few rows whose heads are spread over several."""
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(rows)
    rope = rotary.Rotary(16, base=500.0)
    x = torch.randn((rows, heads + kv, 48), generator=g).to(torch.bfloat16).cuda()
    positions = torch.randint(0, 1 << 20, (rows,), generator=g).int().cuda()
    check(rope, positions, x[:, :heads], x[:, heads:] if kv else None)


@gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("act,rows,heads,kv,dim,rot,start", [
    (torch.bfloat16, 4099, 16, 2, 128, 128, 0), (torch.float16, 40001, 1, 1, 128, 128, 0),
    (torch.float32, 4097, 7, 2, 160, 64, 32), (torch.bfloat16, 9001, 4, 1, 256, 64, 192)], ids=str)
def test_large_calls(act, rows, heads, kv, dim, rot, start, layout):
    """Above 16 MB results are written past the caches.  To the bit what the same rows get in smaller calls, in
    place and apart, and some of them against the definition."""
    from paper_2609_08450_amd import rotary

    assert rows * (heads + kv) * dim * torch.finfo(act).bits // 8 > 16 << 20
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, heads + kv, dim), generator=g, device="cuda").to(act)
    positions = torch.randint(0, 1 << 20, (rows,), generator=g, device="cuda", dtype=torch.int32)
    rope = rotary.Rotary(rot, layout=layout, start=start)
    for transposed in (False, True):
        small = [rotary.rotate(rope, positions[i:i + 800], x[i:i + 800, :heads], x[i:i + 800, heads:], transposed=transposed)
                 for i in range(0, rows, 800)]
        ref = [torch.cat(part) for part in zip(*small)]
        apart = rotary.rotate(rope, positions, x[:, :heads], x[:, heads:], transposed=transposed)
        y = x.clone()
        q, k = y[:, :heads], y[:, heads:]
        rotary.rotate(rope, positions, q, k, q_out=q, k_out=k, transposed=transposed)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(apart, ref)) and all(torch.equal(a, b) for a, b in zip((q, k), ref))
        some = [0, 1, 799, rows // 2, rows - 2, rows - 1]
        want = rotated(unsigned(rope), 1.0, positions[some].tolist(), x[some, :heads].cpu(), start, layout == "interleaved",
                       transposed)
        assert_rotated(apart[0][some], want, 1.0)


@gpu
def test_no_rows():
    from paper_2609_08450_amd import rotary

    rope = rotary.Rotary(16)
    q = torch.empty((0, 4, 16), device="cuda")
    assert rotary.rotate(rope, torch.empty(0, dtype=torch.int32, device="cuda"), q).shape == q.shape


@gpu
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64], ids=str)
def test_far_and_negative_positions(dtype):
    """Whole numbers times whole turns: no position is far."""
    from paper_2609_08450_amd import rotary

    far = [2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, -1, -77777] + ([2 ** 62 + 12345, -2 ** 63] if dtype is torch.int64 else [])
    g = torch.Generator().manual_seed(1)
    q = torch.randn((len(far), 2, 64), generator=g).cuda()
    for rope in (rotary.Rotary(64), rotary.Rotary.of([3.0, 2 * math.pi, math.pi / 2, 1e-9, 0.0, -0.3, 100.0], start=8)):
        check(rope, torch.tensor(far, dtype=dtype).cuda(), q)


@gpu
@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
                                     dict(scaling="yarn", factor=16.0, original=4096), dict(magnitude=0.0),
                                     dict(scaling="bands", factor=8.0, original=8192)], ids=str)
def test_scaled_frequencies(scaling):
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(2)
    rope = rotary.Rotary(128, **scaling)
    q = torch.randn((4, 3, 128), generator=g).cuda()
    check(rope, torch.tensor([0, 77, 31000, 131071], dtype=torch.int32).cuda(), q)
    check(rope, torch.tensor([0, 77, 31000, 131071], dtype=torch.int32).cuda(), q, transposed=True)


@gpu
@pytest.mark.parametrize("off", [0, 1, 2, 4])
def test_strides_alignment_and_surroundings(off):
    """Queries and keys inside a wider buffer, in place and not, at any alignment: what lies around stays."""
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(3)
    flat = torch.randn(7 * 10 * 72 + 16, generator=g).to(torch.bfloat16).cuda()
    rope = rotary.Rotary(32, start=16, layout="interleaved")
    positions = torch.arange(7, dtype=torch.int32).cuda() * 1000

    def parts(x):
        wide = x[off:off + 7 * 10 * 72].view(7, 10, 72)
        return wide[:, 1:5, :64], wide[:, 6:8, 8:]

    q, k = parts(flat)
    ref = [rotated(unsigned(rope), 1.0, positions.tolist(), x.cpu(), 16, True) for x in (q, k)]
    for place in ("in", "other"):
        x = flat.clone()
        to = x if place == "in" else torch.full_like(flat, 3.0)
        before = to.clone()
        (a, b), (c, d) = parts(x), parts(to)
        rotary.rotate(rope, positions, a, b, q_out=c, k_out=d)
        torch.cuda.synchronize()
        assert_rotated(c, ref[0], 1.0, place)
        assert_rotated(d, ref[1], 1.0, place)
        for y in parts(to) + parts(before):
            y.zero_()
        assert torch.equal(to, before), place
        if place == "other":
            assert torch.equal(x, flat)


@gpu
def test_in_place_of_one_and_apart_of_the_other():
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(4)
    q, k = torch.randn((9, 4, 40), generator=g).cuda(), torch.randn((9, 2, 40), generator=g).cuda()
    rope = rotary.Rotary(24, start=4)
    positions = torch.arange(9).cuda()
    ref = [rotated(unsigned(rope), 1.0, positions.tolist(), x.cpu(), 4, False) for x in (q, k)]
    _, out = rotary.rotate(rope, positions, q, k, q_out=q)
    torch.cuda.synchronize()
    assert_rotated(q, ref[0], 1.0)
    assert_rotated(out, ref[1], 1.0)


@gpu
def test_transposed_is_the_gradient():
    """Against the formula's gradient in 64 bits, and against differences: the map is linear, so a step of any
    size has an exact quotient but for the outputs' rounding (2^-24 of each, and the cosines' 2^-21)."""
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(5)
    rope = rotary.Rotary(32, layout="interleaved", start=8, scaling="yarn", factor=8.0, original=512)
    positions = torch.tensor([3, 1000, 123456], dtype=torch.int32).cuda()
    x, dy = (torch.randn((3, 2, 48), generator=g).cuda() for _ in range(2))
    dx = rotary.rotate(rope, positions, dy, transposed=True)

    leaf = x.cpu().double().requires_grad_()
    freq = torch.tensor(unsigned(rope), dtype=torch.float64) * 2.0 ** -64
    angle = 2 * math.pi * torch.remainder(positions.cpu().double()[:, None] * freq, 1.0)
    c, s = rope.magnitude * angle.cos()[:, None], rope.magnitude * angle.sin()[:, None]
    u, v = leaf[..., 8:40:2], leaf[..., 9:40:2]
    y = torch.cat([leaf[..., :8], torch.stack([u * c - v * s, u * s + v * c], -1).flatten(-2), leaf[..., 40:]], -1)
    y.backward(dy.cpu().double())
    # (angles in 64 bits here: off by 2^-53 of a position's turns, far below)
    off = (dx.cpu().double() - leaf.grad).abs()
    assert bool((off <= 2.0 ** -20 * rope.magnitude * 2 * dy.abs().max().cpu()).all())

    for where in ((0, 0, 8), (1, 1, 21), (2, 0, 39), (2, 1, 47)):
        step = x.clone()
        step[where] += 2.0
        moved = rotary.rotate(rope, positions, step).double() - rotary.rotate(rope, positions, x).double()
        slope = float((moved * dy.double()).sum()) / float(step[where].double() - x[where].double())
        size = float(x[where].abs()) + 2 + float(x.abs().max())
        tol = 4 * 2.0 ** -20 * rope.magnitude * size * float(dy.abs().max()) + 2.0 ** -20 * rope.magnitude * 2 * float(dy.abs().max())
        assert abs(slope - float(dx[where])) <= tol, where


@gpu
def test_captured_and_on_other_streams():
    from paper_2609_08450_amd import rotary

    g = torch.Generator().manual_seed(6)
    rope = rotary.Rotary(64)
    q, k = torch.randn((33, 4, 64), generator=g).half().cuda(), torch.randn((33, 1, 64), generator=g).half().cuda()
    positions = torch.arange(33, dtype=torch.int32).cuda()
    ref = rotary.rotate(rope, positions, q, k)
    out = torch.empty_like(q), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = rotary.rotate(rope, positions, q, k, stream=stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rotary.rotate(rope, positions, q, k, q_out=out[0], k_out=out[1])
    for i in range(3):
        positions.add_(7 * i)
        q.mul_(-1)
        ref = rotary.rotate(rope, positions, q, k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), i


# Frequencies, on the CPU.

def test_frequencies_of_each_scaling():
    from paper_2609_08450_amd import rotary

    plain, m = rotary.frequencies(128)
    assert m == 1.0 and plain[0] == 1.0 and math.isclose(plain[-1], 10000.0 ** (-126 / 128))
    linear, _ = rotary.frequencies(128, scaling="linear", factor=4.0)
    assert all(math.isclose(4 * a, b) for a, b in zip(linear, plain))
    ntk, _ = rotary.frequencies(128, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and math.isclose(ntk[-1] * 4, plain[-1])
    yarn, m = rotary.frequencies(128, scaling="yarn", factor=4.0, original=4096)
    assert math.isclose(m, 0.1 * math.log(4) + 1) and rotary.frequencies(8, scaling="yarn", factor=0.5, original=64)[1] == 1.0
    assert yarn[:20] == plain[:20] and math.isclose(4 * yarn[-1], plain[-1])
    bands, m = rotary.frequencies(128, scaling="bands", factor=4.0, original=4096)
    assert m == 1.0
    for f, got in zip(plain, bands):
        turns = 4096 * f / (2 * math.pi)
        if turns >= 4 or turns <= 1:
            assert math.isclose(got, f if turns >= 4 else f / 4)
        else:
            assert f / 4 < got < f
    for x in (yarn, bands):
        assert all(f / 4 <= y * (1 + 1e-12) and y <= f * (1 + 1e-12) for f, y in zip(plain, x))
        assert all(a > b for a, b in zip(x, x[1:]))


def test_turns_are_the_frequencies_to_64_bits():
    from paper_2609_08450_amd import rotary

    f = [1.0, 0.1, 2 * math.pi, 7.0, -0.25, 1e-12, 0.0]
    rope = rotary.Rotary.of(f, device="cpu")
    for x, t in zip(f, rope.turns.tolist()):
        turn = (x / (2 * math.pi)) % 1.0
        d = abs((t % 2 ** 64) / 2.0 ** 64 - turn)
        assert min(d, 1 - d) <= 2.0 ** -53


def test_refused_frequencies():
    from paper_2609_08450_amd import rotary

    for bad in (dict(rot=3), dict(rot=0), dict(rot=8, base=0.0), dict(rot=8, base=math.inf), dict(rot=8, scaling="other"),
                dict(rot=8, scaling="linear", factor=0.0), dict(rot=8, scaling="linear", factor=math.nan),
                dict(rot=2, scaling="ntk", factor=2.0), dict(rot=8, scaling="yarn", factor=2.0),
                dict(rot=8, scaling="bands", factor=2.0), dict(rot=8, scaling="yarn", factor=2.0, original=64, base=1.0),
                dict(rot=8, scaling="yarn", factor=2.0, original=64, slow=40.0),
                dict(rot=8, scaling="bands", factor=2.0, original=64, low=5.0), dict(rot=8, layout="other"),
                dict(rot=8, start=-1), dict(rot=8, magnitude=math.nan), dict(rot=1026)):
        with pytest.raises(rotary.PagedError):
            rotary.Rotary(**bad, device="cpu")
    with pytest.raises(rotary.PagedError):
        rotary.Rotary.of([math.inf], device="cpu")
    with pytest.raises(rotary.PagedError):
        rotary.Rotary.of([], device="cpu")
