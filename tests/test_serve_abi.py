"""CPU checks of libserve_step.so and its bindings: exports, structures, refusals on the host (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "serve_step.h")
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -4
TEXT = open(HEADER).read()


@pytest.fixture(scope="module")
def serve():
    from paper_2609_08450_amd import _serve
    from paper_2609_08450_amd.build import SERVE_LIB_PATH

    if not os.path.exists(SERVE_LIB_PATH):
        pytest.fail("libserve_step.so is not built (run __graft_entry__.build())")
    return _serve


def test_every_declared_symbol_is_exported(serve):
    text = re.sub(r"/\*.*?\*/", "", TEXT, flags=re.S)
    names = sorted(set(re.findall(r"\b(serve_\w+)\s*\(", text)))
    assert names == ["serve_adjust", "serve_compact", "serve_keep", "serve_rotate", "serve_weigh", "serve_weigh_workspace"]
    for name in names:
        assert hasattr(serve.lib(), name), name


@pytest.mark.parametrize("name,mirror", [("serve_rotary", "Rotary"), ("serve_heads", "Heads"), ("serve_lists", "Lists")])
def test_structures_mirror_the_header(serve, name, mirror):
    """Field names and types, in order."""
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), TEXT, flags=re.S).group(1)
    fields = []
    for line in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";"):
        line = line.strip()
        if line:
            base, rest = re.match(r"((?:const )?\w+) (.*)", line, flags=re.S).groups()
            for f in rest.split(","):
                f = f.strip()
                fields.append((f.lstrip("* "), "pointer" if f.startswith("*") else base))
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "pointer": ctypes.c_void_p}
    assert [(n, kinds[k]) for n, k in fields] == [(n.rstrip("_"), t) for n, t in getattr(serve, mirror)._fields_]


def test_packed_structures_are_the_same_bytes(serve):
    heads = (1 << 40, 3, -4, 5, 6, 7, 8)
    assert serve.pack_heads(*heads) == bytes(serve.Heads(*heads))
    lists = (1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13)
    assert serve.pack_lists(*lists) == bytes(serve.Lists(*lists))


def test_constants_mirror_the_header(serve):
    assert serve.ACTS[torch.float32] == int(re.search(r"#define SERVE_F32 (\d+)", TEXT).group(1))
    assert len(serve.ACTS) == 3


P = 4096


def rotate(serve, act=0, turns=P, magnitude=1.0, rot=32, start=0, il=0, positions=P, wide=0, rows=5, dim=64, q=None, k=None):
    def heads(h):
        f = dict(in_=P, in_row=256, in_head=64, out=P, out_row=256, out_head=64, heads=4)
        f.update(h)
        return ctypes.byref(serve.Heads(*(f[n] for n, _ in serve.Heads._fields_)))

    r = serve.Rotary(turns, magnitude, rot, start, il)
    return serve.lib().serve_rotate(act, ctypes.byref(r), positions, wide, rows, dim, heads(q or {}),
                                    heads(k) if k is not None else None, 0, None)


def test_rotate_refusals(serve):
    for bad in (dict(act=3), dict(act=-1), dict(turns=None), dict(turns=4100), dict(magnitude=float("nan")),
                dict(magnitude=float("inf")), dict(rot=0), dict(rot=31), dict(rot=66), dict(start=-1), dict(start=33),
                dict(positions=None), dict(positions=4098), dict(positions=4100, wide=1), dict(rows=-1), dict(dim=0),
                dict(q=dict(heads=0)), dict(k=dict(heads=0)), dict(q=dict(in_=None)), dict(q=dict(out=None)),
                dict(q=dict(in_=4097)), dict(k=dict(out=4097)), dict(act=2, q=dict(in_=4098)),
                dict(q=dict(out_row=512)), dict(k=dict(out_head=32)), dict(rows=1, q=dict(out_head=128))):
        assert rotate(serve, **bad) == EINVAL, bad
    for bad in (dict(rot=1026, dim=2048), dict(dim=65537), dict(q=dict(heads=2 ** 30)), dict(k=dict(heads=2 ** 30))):
        assert rotate(serve, **bad) == EUNSUPPORTED, bad
    assert rotate(serve, rows=0, positions=None) == 0
    L = serve.lib()
    assert L.serve_rotate(0, None, P, 0, 5, 64, None, None, 0, None) == EINVAL


def test_the_angle_s_bound_counts_its_rounding_to_fp32():
    """A rotation's angle is a whole number of 2^-32 turns, rounded down, and its distance from a quarter turn, at most 2^29 of
    them, becomes an FP32 number: the header's bound is of both."""
    rest = torch.arange(2 ** 29 - 2 ** 16, 2 ** 29 + 1, dtype=torch.int64)
    off = 1 + int((rest.float().long() - rest).abs().max())
    about = re.sub(r"[ \n*]+", " ", TEXT[TEXT.index("(a, b) -> m"):TEXT.index("int serve_rotate(")])
    bound = re.search(r"[Aa]ngles are (?:exact to|off by at most) 2\^-(\d+)(?: \+ 2\^-(\d+))? of a turn", about)
    assert off / 2 ** 32 <= sum(2.0 ** -int(x) for x in bound.groups() if x)


def cache_of(**change):
    from paper_2609_08450_amd import paged

    f = dict(k=P, v=None, k_scale=P, v_scale=None, page_stride=2 * 16 * 64, scale_stride=2, n_pages=4, page=16, n_heads=2,
             head_dim=64, code=0)
    f.update(change)
    return ctypes.byref(paged._Cache(*(f[n] for n, _ in paged._Cache._fields_)))


BAD_CACHES = [dict(k=None), dict(k=4100), dict(k_scale=None), dict(n_pages=0), dict(n_heads=0), dict(code=2),
              dict(page_stride=2 * 16 * 64 - 64), dict(page_stride=2 * 16 * 64 + 8), dict(scale_stride=1)]
NO_KERNEL = [dict(page=8), dict(page=48), dict(page=512), dict(head_dim=96, page_stride=2 * 16 * 96),
             dict(n_pages=2 ** 31 - 1, page_stride=64 * 2048)]


def weigh(serve, c=None, act=0, q=P, q_row=256, q_head=64, heads=104, lse=P, table=P, stride=8, width=8, starts=P, n=3, lens=P,
          rows=5, scale=0.1, w=P, offsets=P, ws=P, size=1 << 40):
    return serve.lib().serve_weigh(c or cache_of(), act, q, q_row, q_head, heads, lse, table, stride, width, starts, n, lens,
                                   rows, scale, w, offsets, ws, size, None)


def compact(serve, c=None, table=P, stride=8, width=8, kept=P, kw=5, counts=P, n=3):
    return serve.lib().serve_compact(c or cache_of(), table, stride, width, kept, kw, counts, n, None)


def test_caches_are_checked(serve):
    for change in BAD_CACHES:
        assert weigh(serve, cache_of(**change)) == EINVAL and compact(serve, cache_of(**change)) == EINVAL, change
    for change in NO_KERNEL:
        assert weigh(serve, cache_of(**change)) == EUNSUPPORTED and compact(serve, cache_of(**change)) == EUNSUPPORTED, change
    assert compact(serve, cache_of(v=P)) == EINVAL
    assert weigh(serve, n=0) == 0
    assert serve.lib().serve_compact(None, P, 8, 8, P, 5, P, 3, None) == EINVAL


def test_weigh_refusals(serve):
    for bad in (dict(act=2), dict(act=-1), dict(q=None), dict(q=4100), dict(q_row=250), dict(q_head=4), dict(heads=0),
                dict(heads=103), dict(lse=None), dict(table=None), dict(width=0), dict(stride=7), dict(starts=None),
                dict(lens=None), dict(rows=-1), dict(n=-1), dict(scale=-0.1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(w=None), dict(offsets=None), dict(ws=None), dict(ws=4104)):
        assert weigh(serve, **bad) == EINVAL, bad
    assert weigh(serve, width=2 ** 27, stride=2 ** 27) == EUNSUPPORTED
    assert weigh(serve, rows=0, q=None, ws=None) == 0
    L = serve.lib()
    for sizes in ((-1, 3, 4, 2), (5, -1, 4, 2), (5, 3, 0, 2), (5, 3, 4, 0), (5, 3, 5, 2)):
        assert L.serve_weigh_workspace(*sizes) == 0


def test_scales_past_what_products_are_scaled_by(serve):
    """log2(e) times the scale has to be an FP32 number, too."""
    largest = torch.finfo(torch.float32).max
    for scale in (largest, 2.4e38):
        assert weigh(serve, scale=scale) == EUNSUPPORTED and weigh(serve, scale=scale, rows=0) == EUNSUPPORTED
    assert weigh(serve, scale=2.35e38, rows=0) == 0


def keep(serve, idx=P, K=5, base=0, lens=P, n=3, first=1, last=2, kept=12288, width=8, counts=8192, w=None, offsets=None):
    return serve.lib().serve_keep(idx, K, base, lens, n, first, last, kept, width, counts, w, offsets, None)


def test_keep_and_compact_refusals(serve):
    for bad in (dict(idx=None), dict(K=-1), dict(base=-1), dict(lens=None), dict(n=-1), dict(first=-1), dict(last=-1),
                dict(kept=None), dict(width=7), dict(counts=None), dict(w=P), dict(counts=P), dict(kept=P),
                dict(first=2 ** 31 - 1, last=2 ** 31 - 1, width=2 ** 31 - 1)):
        assert keep(serve, **bad) == EINVAL, bad
    assert keep(serve, n=0, idx=None, lens=None) == 0
    for bad in (dict(table=None), dict(width=0), dict(stride=7), dict(kept=None), dict(kw=-1), dict(counts=None), dict(n=-1)):
        assert compact(serve, **bad) == EINVAL, bad
    for bad in (dict(n=65536), dict(width=2 ** 28, stride=2 ** 28)):
        assert compact(serve, **bad) == EUNSUPPORTED, bad
    assert compact(serve, n=0, table=None) == 0 and compact(serve, kw=0, kept=None) == 0


def adjust(serve, act=0, x=P, x_row=64, out=8192, out_row=64, rows=3, vocab=50, **lists):
    f = {n: None if t is ctypes.c_void_p else 0 for n, t in serve.Lists._fields_}
    f.update(lists)
    s = serve.Lists(*(f[n] for n, _ in serve.Lists._fields_))
    return serve.lib().serve_adjust(act, x, x_row, out, out_row, rows, vocab, ctypes.byref(s), None)


def test_adjust_refusals(serve):
    for bad in (dict(act=3), dict(act=-1), dict(x=None), dict(x=4097), dict(act=2, x=4098), dict(out=None), dict(out=8194),
                dict(rows=-1), dict(vocab=0), dict(x=8192), dict(act=2, x=8192, x_row=60), dict(out_row=49), dict(tokens=P),
                dict(bias_ids=P), dict(bias_ids=P, bias=P), dict(bias_ids=P, bias_starts=P),
                dict(mask=P, mask_stride=1, n_masks=3), dict(mask=P, mask_stride=2, n_masks=-1, row_mask=P),
                dict(mask=P, mask_stride=2, n_masks=2)):
        assert adjust(serve, **bad) == EINVAL, bad
    for bad in (dict(rows=65536), dict(vocab=2 ** 31 - 1, out_row=2 ** 31)):
        assert adjust(serve, **bad) == EUNSUPPORTED, bad
    assert adjust(serve, rows=0, x=None) == 0
    assert serve.lib().serve_adjust(0, P, 64, P, 64, 3, 50, None, None) == EINVAL


def test_bindings_fail_loudly_without_library(serve, tmp_path, monkeypatch):
    monkeypatch.setattr(serve, "SERVE_LIB_PATH", str(tmp_path / "missing.so"))
    monkeypatch.setattr(serve, "_lib", None)
    with pytest.raises(serve.PagedError, match="missing"):
        serve.lib()


# The bindings' own checks.  The devices here are said to be: none of these calls gets as far as the library.

class On0(torch.Tensor):
    def get_device(self):
        return 0


class On1(torch.Tensor):
    def get_device(self):
        return 1


i32, i64, b16, f32 = torch.int32, torch.int64, torch.bfloat16, torch.float32


def signatures():
    """name: module, plain arguments, tensors."""
    weigh = dict(q=(b16, 5, 4, 64), lse=(f32, 5, 4), table=(i32, 3, 8), row_starts=(i32, 4), row_lengths=(i32, 5),
                 weights=(f32, 100), weight_offsets=(i64, 3), workspace=(torch.uint8, 4096))
    return {
        "rotate": ("rotary", {}, dict(positions=(i32, 5), q=(b16, 5, 4, 64), k=(b16, 5, 2, 64), q_out=(b16, 5, 4, 64),
                                      k_out=(b16, 5, 2, 64))),
        "weigh": ("evict", dict(scale=0.1), weigh),
        "keep": ("evict", dict(first=1, last=2), dict(idx=(i32, 3, 7), lens=(i32, 3), kept=(i32, 3, 10), counts=(i32, 3),
                                                      weights=(f32, 3, 50), weight_offsets=(i64, 3))),
        "compact": ("evict", {}, dict(table=(i32, 3, 8), kept=(i32, 3, 10), counts=(i32, 3))),
        "adjust": ("logits", {}, dict(x=(b16, 3, 50), out=(f32, 3, 50), tokens=(i32, 9), token_starts=(i64, 4),
                                      prompt_lens=(i32, 3), repetition=(f32, 3), frequency=(f32, 3), presence=(f32, 3),
                                      bias_ids=(i32, 6), bias=(f32, 6), bias_starts=(i64, 4), mask=(i32, 2, 2),
                                      row_mask=(i32, 3))),
    }


class Reached(Exception):
    pass


class Nothing:
    def serve_weigh_workspace(self, *args):
        return 4096

    def __getattr__(self, name):
        def call(*args):
            raise Reached
        return call


@pytest.fixture
def call(monkeypatch):
    from paper_2609_08450_amd import _serve, evict, logits, paged, rotary

    monkeypatch.setattr(_serve, "_lib", Nothing())
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(paged._topk, "_stream", lambda stream: 0)
    cache = paged.PagedCache.__new__(paged.PagedCache)
    cache.n_heads, cache.head_dim, cache.v, cache._ref, cache._device = 2, 64, None, None, 0
    rope = rotary.Rotary(32, device="cpu")
    rope._device = 0

    def go(name, device=0, where=None, **change):
        monkeypatch.setattr(paged, "_current_device", lambda: device)
        module, plain, tensors = signatures()[name]
        made = {n: torch.zeros(shape, dtype=dtype).as_subclass(On1 if n == where else On0)
                for n, (dtype, *shape) in tensors.items()}
        args = {**plain, **made}
        for n, x in change.items():
            args[n] = x(args[n]).as_subclass(On0) if callable(x) else x
        first = {} if name in ("keep", "adjust") else dict(rotary=rope) if name == "rotate" else dict(cache=cache)
        return getattr({"rotary": rotary, "evict": evict, "logits": logits}[module], name)(**first, **args)

    return go


@pytest.mark.parametrize("name", sorted(signatures()))
def test_tensors_of_another_device_are_refused(call, name):
    from paper_2609_08450_amd import paged

    with pytest.raises(Reached):
        call(name)
    for where in signatures()[name][2]:
        with pytest.raises(paged.PagedError, match="cuda:1"):
            call(name, where=where)
    with pytest.raises(paged.PagedError, match="cuda:1"):
        call(name, device=1)


@pytest.mark.parametrize("name", sorted(signatures()))
def test_other_types_and_shapes_are_refused(call, name):
    """Every tensor: of another type, one axis more, and one entry fewer where its size follows from the others'."""
    from paper_2609_08450_amd import paged

    free = {"weights", "workspace", "bias_ids", "tokens", "kept", "table", "idx", "mask"}  # sizes of their own
    for where, (dtype, *shape) in signatures()[name][2].items():
        with pytest.raises(paged.PagedError):
            call(name, **{where: lambda t: t.to(torch.float64)})
        if where not in ("weights", "workspace"):
            with pytest.raises(paged.PagedError):
                call(name, **{where: lambda t: t[None]})
        if where not in free:
            with pytest.raises(paged.PagedError):
                call(name, **{where: lambda t: t[:-1].contiguous()})


def test_arguments_that_belong_together(call):
    from paper_2609_08450_amd import paged

    for name, change in (
            ("rotate", dict(k=None)), ("rotate", dict(q_out=lambda t: t[:, :1].expand(5, 4, 64))),
            ("rotate", dict(q=lambda t: t.transpose(1, 2).contiguous().transpose(1, 2))),
            ("keep", dict(weights=None)), ("keep", dict(weight_offsets=None)),
            ("adjust", dict(tokens=None)), ("adjust", dict(token_starts=None)), ("adjust", dict(bias=None)),
            ("adjust", dict(bias_ids=None)), ("adjust", dict(bias_starts=None)), ("adjust", dict(mask=None)),
            ("adjust", dict(row_mask=None)), ("adjust", dict(mask=lambda t: t[:, :1].contiguous())),
            ("adjust", dict(tokens=None, token_starts=None)), ("adjust", dict(bias=lambda t: t[:-1])),
            ("adjust", dict(out=lambda t: t[:1].expand(3, 50))),
            ("weigh", dict(q=lambda t: t[..., :32])), ("weigh", dict(lse=lambda t: t.t().contiguous().t())),
            ("compact", dict(table=lambda t: t.t().contiguous().t()))):
        with pytest.raises(paged.PagedError):
            call(name, **change)
    for name, change in (
            ("rotate", dict(k=None, k_out=None)), ("rotate", dict(positions=lambda t: t.long())),
            ("keep", dict(weights=None, weight_offsets=None)),
            ("adjust", dict(bias=None, bias_ids=None, bias_starts=None)), ("adjust", dict(mask=None, row_mask=None)),
            ("adjust", dict(tokens=None, token_starts=None, prompt_lens=None, repetition=None, frequency=None, presence=None))):
        with pytest.raises(Reached):
            call(name, **change)
