"""CPU checks of libpaged_kv.so: it loads, exports every function the header
declares, and refuses bad arguments on the host (no GPU needed)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "paged_kv.h")
EINVAL, EUNSUPPORTED = -1, -2


@pytest.fixture(scope="module")
def paged():
    from paper_2609_08450_amd import paged
    from paper_2609_08450_amd.build import PAGED_LIB_PATH

    if not os.path.exists(PAGED_LIB_PATH):
        pytest.fail("libpaged_kv.so is not built (run __graft_entry__.build())")
    return paged


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(paged_kv_\w+)\s*\(", text)))


def test_every_declared_symbol_is_exported(paged):
    names = declared()
    assert "paged_kv_attend" in names and "paged_kv_tables" in names and len(names) == 7
    for name in names:
        assert hasattr(paged.lib(), name), name


def test_constants_mirror_the_header(paged):
    text = open(HEADER).read()
    value = lambda n: int(re.search(rf"#define {n} \(?(-?\d+)", text).group(1))  # noqa: E731
    assert paged.WORKSPACE_ZEROED == value("PAGED_KV_WORKSPACE_ZEROED")
    assert sorted(paged.CODES.values()) == [value("PAGED_KV_E4M3"), value("PAGED_KV_INT8")]
    assert sorted(paged.ACTS.values()) == [value("PAGED_KV_BF16"), value("PAGED_KV_F16")]


def cache_of(paged, **change):
    f = dict(k=4096, v=4096, k_scale=4096, v_scale=4096, page_stride=2 * 16 * 64, scale_stride=2, n_pages=4, page=16,
             n_heads=2, head_dim=64, code=0)
    f.update(change)
    return ctypes.byref(paged._Cache(*(f[n] for n, _ in paged._Cache._fields_)))


BAD_CACHES = [dict(k=None), dict(k=4100), dict(k_scale=None), dict(n_pages=0), dict(n_heads=0), dict(code=2),
              dict(code=-1), dict(page_stride=2 * 16 * 64 - 64), dict(page_stride=2 * 16 * 64 + 8), dict(scale_stride=1)]
NO_KERNEL = [dict(page=8), dict(page=48), dict(page=512), dict(head_dim=96, page_stride=2 * 16 * 96),
             dict(n_pages=2 ** 31 - 1, page_stride=64 * 2048)]


def calls(paged, c, P=4096, act=0, heads=4, q_row=256, n=3, rows=5, stride=8, width=8, scale=0.1, K=7, ws=4096,
          size=1 << 40):
    L = paged.lib()
    return {
        "store": lambda: L.paged_kv_store(c, act, P, q_row, 64, P, q_row, 64, P, rows, None),
        "attend": lambda: L.paged_kv_attend(c, act, P, q_row, 64, heads, P, stride, width, P, n, P, rows, scale, P, P, ws,
                                            size, None),
        "selected": lambda: L.paged_kv_attend_selected(c, act, P, q_row, 64, heads, P, K, P, stride, width, P, n, P, rows,
                                                       scale, P, P, ws, size, None),
        "score": lambda: L.paged_kv_score(c, act, P, q_row, 64, heads, P, P, stride, width, P, n, P, rows, scale, P, P,
                                          None),
    }


@pytest.mark.parametrize("change", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(paged, change):
    for name, call in calls(paged, cache_of(paged, **change)).items():
        assert call() == EINVAL, name


@pytest.mark.parametrize("change", NO_KERNEL, ids=str)
def test_caches_without_a_kernel_are_refused(paged, change):
    for name, call in calls(paged, cache_of(paged, **change)).items():
        assert call() == EUNSUPPORTED, name


def test_bad_arguments_are_refused(paged):
    c = cache_of(paged)
    for change in (dict(act=2), dict(act=-1), dict(rows=-1), dict(P=None), dict(P=4100), dict(q_row=250)):
        for name, call in calls(paged, c, **change).items():
            assert call() == EINVAL, (change, name)
    for change in (dict(heads=0), dict(heads=3), dict(n=-1), dict(width=0), dict(stride=7), dict(ws=None), dict(ws=4104),
                   dict(scale=-0.1), dict(scale=float("nan")), dict(scale=float("inf"))):
        for name, call in calls(paged, c, **change).items():
            if name in ("store", "score"):
                continue
            assert call() == EINVAL, (change, name)
    one = cache_of(paged, n_heads=1, v=None, v_scale=None)
    assert calls(paged, one, heads=0)["score"]() == EINVAL
    assert calls(paged, one, width=0)["score"]() == EINVAL
    assert calls(paged, one, heads=129)["score"]() == EUNSUPPORTED
    assert calls(paged, c)["score"]() == EUNSUPPORTED                   # a cache of two heads
    assert calls(paged, c, K=0)["selected"]() == EINVAL
    assert calls(paged, c, K=2 ** 31 - 1)["selected"]() == EUNSUPPORTED
    far = calls(paged, c, width=2 ** 27, stride=2 ** 27)                # more tokens than 32 bits count
    assert far["attend"]() == EUNSUPPORTED and far["selected"]() == EUNSUPPORTED
    assert calls(paged, one)["attend"]() == EINVAL                      # no values
    assert calls(paged, one)["store"]() == EINVAL                       # v_new without values
    # nothing to do is no error, whatever the pointers
    for name, call in calls(paged, c, P=None, rows=0, ws=None).items():
        assert call() == 0, name


def test_tables_arguments(paged):
    def call(ring=4096, size=16, n=3, table=4096, stride=8, width=8, page=16, rows=5, lens_out=8192, slots=4096):
        return paged.lib().paged_kv_tables(ring, size, 4096, 4096, 4096, 4096, lens_out, n, table, stride, width, page,
                                           rows, 4096, 4096, 4096, slots, None)

    for bad in (dict(ring=None), dict(size=0), dict(n=-1), dict(table=None), dict(stride=7), dict(width=0),
                dict(rows=-1), dict(lens_out=4096), dict(lens_out=None), dict(slots=None)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(page=8), dict(page=24), dict(width=2 ** 28, stride=2 ** 28)):
        assert call(**bad) == EUNSUPPORTED, bad


def test_the_header_says_which_tables_arguments_may_be_one(paged):
    text = " ".join(open(HEADER).read().replace("*", " ").split())

    def call(pool_out, lens_out, n):  # nothing is launched here: without a GPU the last check refuses
        return paged.lib().paged_kv_tables(4096, 16, 4096, pool_out, 4096, 4096, lens_out, n, 4096, 8, 8, 16, 0, 4096,
                                           None, None, None, None)

    assert "pool_out may be pool_in." in text and "lens_out may not be lens_in (EINVAL)" in text
    assert "lens_out may be lens_in" not in text
    assert call(8192, 4096, 3) == EINVAL
    import torch

    if not torch.cuda.is_available():
        assert call(4096, 8192, 3) == EUNSUPPORTED


def test_status_texts(paged):
    L = paged.lib()
    assert L.paged_kv_status_str(-1) == b"invalid argument"
    assert L.paged_kv_status_str(-4) == b"workspace too small"
    assert L.paged_kv_status_str(-99) == b"unknown status"


def test_binding_refuses_host_tensors(paged):
    import torch

    x = torch.zeros((2, 1, 16, 64), dtype=torch.int8)
    with pytest.raises(paged.PagedError, match="device"):
        paged.PagedCache.of(x, torch.ones((2, 1)), x, torch.ones((2, 1)))
    with pytest.raises(paged.PagedError, match="device"):
        paged.tables(torch.zeros(4, dtype=torch.int32), None, torch.zeros(1), None, torch.zeros((1, 1)), 16, pool_out=None,
                     lens_out=None, row_starts=None, row_request=None, row_lengths=None, slots=torch.zeros(1))


def test_binding_fails_loudly_without_library(paged, tmp_path, monkeypatch):
    monkeypatch.setattr(paged, "PAGED_LIB_PATH", str(tmp_path / "missing.so"))
    monkeypatch.setattr(paged, "_lib", None)
    with pytest.raises(paged.PagedError):
        paged.lib()
