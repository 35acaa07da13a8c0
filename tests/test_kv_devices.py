"""The operators on KV blocks take tensors of the current device alone."""
import types

import pytest
import torch

import paper_2411_03357_amd as pgcm
from paper_2411_03357_amd import kv


class _Elsewhere:
    """a tensor of a second GPU, as far as it is looked at"""
    is_cuda = True

    def __init__(self, like):
        self.shape, self.dtype, self.stride, self.dim, self.is_contiguous = (
            torch.Size(like.shape), like.dtype, like.stride, like.dim, like.is_contiguous)

    def get_device(self):
        return 1

    def data_ptr(self):
        raise AssertionError("not to be asked")


def _calls(make, cache):
    i32 = lambda *shape: make(torch.zeros(shape, dtype=torch.int32))
    f32 = lambda *shape: make(torch.zeros(shape))
    half = lambda *shape: make(torch.zeros(shape, dtype=torch.float16))
    i64, i8 = make(torch.zeros(2, dtype=torch.int64)), make(torch.zeros(4, 2, 2, 64, dtype=torch.int8))
    space = types.SimpleNamespace(_h=None)
    return {
        "append": lambda: pgcm.kv_append(cache, half(2, 4, 64), half(2, 2, 64), half(2, 2, 64), None, i64, half(2, 4, 64), stream=0),
        "attend": lambda: pgcm.kv_attend(cache, half(2, 4, 64), i32(2, 3), i32(2), half(2, 4, 64), workspace=space, stream=0),
        "summarize": lambda: pgcm.kv_summarize(cache, i32(2), i32(2), i8, f32(4, 2), stream=0),
        "select": lambda: pgcm.kv_select(half(2, 4, 64), i32(2, 3), i32(2), i8, f32(4, 2), 16, i32(2, 2, 1), workspace=space,
                                         stream=0),
        "evict": lambda: pgcm.kv_evict(f32(2, 3), i32(2, 3), i32(2), 16, i32(2), i32(2, 1), stream=0),
    }


@pytest.mark.parametrize("op", ["append", "attend", "summarize", "select", "evict"])
@pytest.mark.parametrize("cache_on", [0, 1])
def test_tensors_and_caches_of_another_device_are_refused(monkeypatch, op, cache_on):
    monkeypatch.setattr(kv, "_device", lambda: 0)
    c = kv._Placed(kv._Cache(1 << 20, 1 << 20, 0, 4, 16, 2, 64, 0, 2048, 128, 64, 2048, 128, 64), cache_on)
    cache = types.SimpleNamespace(_c=c, _at=kv.C.addressof(c), device=cache_on, kv_heads=2, head_dim=64, dtype=torch.float16)
    with pytest.raises(ValueError, match="is on cuda:1, and the current device is cuda:0"):
        _calls(_Elsewhere, cache)[op]()


@pytest.mark.gpu
@pytest.mark.parametrize("op", ["append", "attend", "summarize", "select", "evict"])
def test_the_native_marshalling_compares_devices(monkeypatch, op):
    pool = torch.zeros(4, 2, 16, 2, 64, dtype=torch.float16, device="cuda")
    cache = pgcm.KVCache(pool[:, 0], pool[:, 1])
    call = _calls(lambda t: t.cuda(), cache)[op]
    monkeypatch.setattr(pgcm.kv, "_device", lambda: 1)      # as if another device were the current one
    given = []
    native = kv._native()
    watched = types.SimpleNamespace(**{"kv_" + n: lambda *a, n=n: given.append(getattr(native, "kv_" + n)(1, *a[1:])) or given[-1]
                                       for n in ("append", "attend", "summarize", "select", "evict")})
    monkeypatch.setattr(kv, "_marshal", watched)
    with pytest.raises(ValueError, match="is on cuda:0, and the current device is cuda:1"):
        call()
    assert given == [None]
