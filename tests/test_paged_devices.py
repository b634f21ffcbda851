"""Every tensor of a paged call lies on one device, the current one.  The devices here are
said to be: none of these calls gets as far as the library."""
import pytest
import torch

from paper_2609_08450_amd import paged


class On0(torch.Tensor):
    def get_device(self):
        return 0


class On1(torch.Tensor):
    def get_device(self):
        return 1


i32, i64, b16, f32 = torch.int32, torch.int64, torch.bfloat16, torch.float32


def shapes():
    tables = dict(ring=(i32, 40), pool=(i32, 4), lens=(i32, 3), new_lens=(i32, 3), table=(i32, 3, 8), pool_out=(i32, 4),
                  lens_out=(i32, 3), row_starts=(i32, 4), row_request=(i32, 5), row_lengths=(i32, 5), slots=(i64, 5))
    q = dict(q=(b16, 5, 4, 64), table=(i32, 3, 8))
    return {
        "tables": (dict(page=16), tables),
        "store": ({}, dict(k_new=(b16, 5, 2, 64), v_new=(b16, 5, 2, 64), slots=(i64, 5))),
        "attend": (dict(scale=0.1), dict(q, row_starts=(i32, 4), row_lengths=(i32, 5), out=(b16, 5, 4, 64), lse=(f32, 5, 4),
                                         workspace=(torch.uint8, 4096))),
        "attend_selected": (dict(scale=0.1), dict(q, idx=(i32, 5, 7), row_request=(i32, 5), row_lengths=(i32, 5),
                                                  out=(b16, 5, 4, 64), lse=(f32, 5, 4), workspace=(torch.uint8, 4096))),
        "score": (dict(scale=0.1), dict(q, w=(f32, 5, 4), row_request=(i32, 5), row_lengths=(i32, 5), scores=(f32, 100),
                                        row_offsets=(i64, 5))),
    }


class Reached(Exception):
    pass


class Nothing:
    def __getattr__(self, name):
        def call(*args):
            raise Reached
        return call


@pytest.mark.parametrize("name", sorted(shapes()))
def test_tensors_of_another_device_are_refused(name, monkeypatch):
    monkeypatch.setattr(paged, "_lib", Nothing())
    monkeypatch.setattr(paged, "_current_device", lambda: 0)
    monkeypatch.setattr(paged._topk, "_stream", lambda stream: 0)
    monkeypatch.setattr(paged.PagedCache, "workspace_size", lambda self, *sizes: 4096)
    cache = paged.PagedCache.__new__(paged.PagedCache)
    cache.n_heads, cache.head_dim, cache.v, cache._ref, cache._device = 2, 64, True, None, 0
    plain, tensors = shapes()[name]
    first = {} if name == "tables" else dict(cache=cache)

    def call(where, device=0):
        monkeypatch.setattr(paged, "_current_device", lambda: device)
        made = {n: torch.zeros(shape, dtype=dtype).as_subclass(On1 if n == where else On0)
                for n, (dtype, *shape) in tensors.items()}
        getattr(paged, name)(**first, **plain, **made)

    with pytest.raises(Reached):
        call(None)
    for where in tensors:
        with pytest.raises(paged.PagedError, match="cuda:1"):
            call(where)
    with pytest.raises(paged.PagedError, match="current device is cuda:1"):
        call(None, device=1)
