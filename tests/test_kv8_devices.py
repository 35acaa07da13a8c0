"""The operators on KV blocks in 8 bits take tensors of the current device alone, named or native."""
import types

import pytest
import torch

import paper_2411_03357_amd as pgcm
from paper_2411_03357_amd import kv, kv8
from test_kv_devices import _Elsewhere

OPS = ["kv8_append", "kv8_store", "kv8_load", "kv8_attend", "kv_window"]


def _calls(make, cache8, cache):
    i32 = lambda *shape: make(torch.zeros(shape, dtype=torch.int32))
    half = lambda *shape: make(torch.zeros(shape, dtype=torch.float16))
    i64 = make(torch.zeros(2, dtype=torch.int64))
    space = types.SimpleNamespace(_h=None)
    attend = lambda call, c: lambda: call(c, half(2, 4, 64), i32(2, 3), i32(2), half(2, 4, 64), workspace=space, stream=0)
    return {
        "kv8_append": lambda: pgcm.kv8_append(cache8, half(2, 4, 64), half(2, 2, 64), half(2, 2, 64), None, i64, half(2, 4, 64),
                                              stream=0),
        "kv8_store": lambda: pgcm.kv8_store(cache8, cache, i32(2), i32(2), stream=0),
        "kv8_load": lambda: pgcm.kv8_load(cache8, cache, i32(2), i32(2), i32(2), stream=0),
        "kv8_attend": attend(pgcm.kv8_attend, cache8),
        "kv_window": attend(pgcm.kv_window, cache),
    }


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("cache_on", [0, 1])
def test_tensors_and_caches_of_another_device_are_refused(monkeypatch, op, cache_on):
    monkeypatch.setattr(kv, "_device", lambda: 0)
    at = 1 << 20
    c8 = kv8._Placed8(kv8._Cache8(at, at, at, at, 0, 0, 4, 16, 2, 64, 2048, 128, 64, 2048, 128, 64, 2, 1, 2, 1), cache_on)
    c = kv._Placed(kv._Cache(at, at, 0, 4, 16, 2, 64, 0, 2048, 128, 64, 2048, 128, 64), cache_on)
    of = lambda c: types.SimpleNamespace(_c=c, _at=kv.C.addressof(c), device=cache_on, kv_heads=2, head_dim=64, dtype=torch.float16)
    with pytest.raises(ValueError, match="is on cuda:1, and the current device is cuda:0"):
        _calls(_Elsewhere, of(c8), of(c))[op]()


@pytest.mark.gpu
@pytest.mark.parametrize("op", OPS)
def test_the_native_marshalling_compares_devices(monkeypatch, op):
    pool = torch.zeros(4, 2, 16, 2, 64, dtype=torch.float16, device="cuda")
    codes, scales = torch.zeros(4, 2, 16, 2, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, 2, 2, device="cuda")
    cache8 = pgcm.KV8Cache(codes[:, 0], codes[:, 1], scales[:, 0], scales[:, 1], torch.float16)
    call = _calls(lambda t: t.cuda(), cache8, pgcm.KVCache(pool[:, 0], pool[:, 1]))[op]
    monkeypatch.setattr(kv, "_device", lambda: 1)      # as if another device were the current one
    given = []
    native = kv8._native()
    watched = types.SimpleNamespace(**{n: lambda *a, n=n: given.append(getattr(native, n)(1, *a[1:])) or given[-1] for n in OPS})
    monkeypatch.setattr(kv8, "_marshal", watched)
    with pytest.raises(ValueError, match="is on cuda:0, and the current device is cuda:1"):
        call()
    assert given == [None]
