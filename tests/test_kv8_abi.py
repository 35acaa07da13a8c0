"""The C ABI of the operators on KV blocks in 8 bits: exported, and arguments refused before anything reaches the GPU."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import paper_2411_03357_amd as pgcm
from paper_2411_03357_amd import kv, kv8
import kv8_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, ALIGN = -1, -2
AT = 1 << 20            # an address; no call here gets as far as using it


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "pgcm_kv8.h")).read()
    names = sorted(set(re.findall(r"\b(pgcm_kv8?_[a-z_0-9]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(pgcm.KV8_EXPORTS) == names
    lib = C.CDLL(pgcm.library_path())
    for n in names:
        assert hasattr(lib, n), n


def _cache8(**change):
    c = kv8._Cache8(AT, AT, AT, AT, 0, 0, 10, 16, 2, 128, 8192, 256, 128, 8192, 256, 128, 2, 1, 2, 1)
    for name, value in change.items():
        setattr(c, name, value)
    return c


def _cache(**change):
    c = kv._Cache(AT, AT, 0, 10, 16, 2, 128, 0, 8192, 256, 128, 8192, 256, 128)
    for name, value in change.items():
        setattr(c, name, value)
    return c


def _append(**change):
    a = kv._Append(5, 4, AT, AT, AT, 512, 128, 256, 128, 256, 128, AT, AT, AT, AT, 1e-6, 0, AT, 100, 128, AT, 512, 128)
    for name, value in change.items():
        setattr(a, name, value)
    return a


BAD_CACHES = [dict(k=None), dict(v=None), dict(k_scales=None), dict(v_scales=None), dict(code=2), dict(half=2), dict(blocks=0),
              dict(blocks=1 << 31), dict(block_tokens=0), dict(block_tokens=8), dict(block_tokens=24), dict(block_tokens=4112),
              dict(kv_heads=0), dict(kv_heads=70000), dict(head_dim=0), dict(head_dim=8), dict(head_dim=72), dict(head_dim=272)]
UNALIGNED_CACHES = [dict(k=AT + 8), dict(v=AT + 1), dict(k_block=8), dict(k_token=129), dict(k_head=-4), dict(v_block=1),
                    dict(v_token=24), dict(v_head=2), dict(k_scales=AT + 2), dict(v_scales=AT + 1)]


def test_caches_are_refused():
    lib = kv8._lib()
    for bad, status in [(b, ARG) for b in BAD_CACHES] + [(b, ALIGN) for b in UNALIGNED_CACHES]:
        at = C.addressof(cache := _cache8(**bad))
        assert lib.pgcm_kv8_append(at, C.byref(_append()), None) == status, bad
        for move in (lib.pgcm_kv8_store, lib.pgcm_kv8_load):
            assert move(at, C.byref(_cache()), 3, AT, AT, None, None) == status, bad
        del cache
    for bad, status in ((dict(k=None), ARG), (dict(blocks=0), ARG), (dict(reserved=1), ARG), (dict(k=AT + 8), ALIGN),
                        # not as the other cache
                        (dict(half=1), ARG), (dict(block_tokens=32), ARG), (dict(kv_heads=3), ARG), (dict(head_dim=64), ARG)):
        for move in (lib.pgcm_kv8_store, lib.pgcm_kv8_load):
            assert move(C.byref(_cache8()), C.byref(_cache(**bad)), 3, AT, AT, None, None) == status, bad


def test_moves_refuse():
    lib, c8, c = kv8._lib(), _cache8(), _cache()
    for move in (lib.pgcm_kv8_store, lib.pgcm_kv8_load):
        assert move(None, C.byref(c), 3, AT, AT, None, None) == ARG
        assert move(C.byref(c8), None, 3, AT, AT, None, None) == ARG
        assert move(C.byref(c8), C.byref(c), 3, None, AT, None, None) == ARG
        assert move(C.byref(c8), C.byref(c), 1 << 31, AT, AT, None, None) == ARG
        assert move(C.byref(c8), C.byref(c), (1 << 31) - 1, AT, AT, None, None) == ARG      # more than a launch holds
        assert move(C.byref(c8), C.byref(c), 0, None, None, None, None) == 0


def test_append_refuses():
    lib, cache = kv8._lib(), _cache8()
    at = C.addressof(cache)
    assert lib.pgcm_kv8_append(at, None, None) == ARG and lib.pgcm_kv8_append(None, C.byref(_append()), None) == ARG
    for bad in (dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None),
                dict(heads=3), dict(heads=0), dict(heads=70000), dict(eps=-1.0), dict(eps=math.nan), dict(rope_dim=0),
                dict(rope_dim=24), dict(rope_dim=144), dict(rope_positions=0), dict(tokens=1 << 31), dict(tokens=(1 << 31) - 1),
                dict(k_token=-256), dict(v_token=(1 << 23) + 8)):
        assert lib.pgcm_kv8_append(at, C.byref(_append(**bad)), None) == ARG, bad
    for bad in (dict(q=AT + 2), dict(k=AT + 2), dict(v=AT + 2), dict(q_out=AT + 2), dict(q_token=3), dict(q_head=3),
                dict(k_token=3), dict(k_head=3), dict(v_token=3), dict(v_head=3), dict(q_out_token=3), dict(q_out_head=3),
                dict(q_weight=AT + 2), dict(k_weight=AT + 2), dict(rope=AT + 4)):
        assert lib.pgcm_kv8_append(at, C.byref(_append(**bad)), None) == ALIGN, bad
    for bad in (dict(k_token=(1 << 23) + 16), dict(v_token=-16)):
        assert lib.pgcm_kv8_append(C.byref(_cache8(**bad)), C.byref(_append()), None) == ARG, bad
    assert lib.pgcm_kv8_append(at, C.byref(_append(tokens=0, k=None)), None) == 0


def _window(**change):
    a = kv8._Window(3, 4, 5, 3, AT, AT, 512, 128, AT, 20, 20, 0.1, AT, 100, 4, AT, 512, 128, None)
    for name, value in change.items():
        setattr(a, name, value)
    return a


def test_attention_refuses():
    lib, some = kv8._lib(), C.create_string_buffer(256)
    for call, cache, other in ((lib.pgcm_kv8_attend, _cache8, BAD_CACHES + UNALIGNED_CACHES),
                               (lib.pgcm_kv_window, _cache, [dict(k=None), dict(half=2), dict(reserved=1), dict(v=AT + 8)])):
        good = cache()
        at = C.addressof(good)
        assert call(None, at, C.byref(_window()), None) == ARG
        assert call(some, None, C.byref(_window()), None) == ARG
        assert call(some, at, None, None) == ARG
        for bad in other:
            assert call(some, C.byref(cache(**bad)), C.byref(_window()), None) in (ARG, ALIGN), bad
        for bad in (dict(q=None), dict(out=None), dict(lens=None), dict(tables=None), dict(scale=math.nan), dict(scale=math.inf),
                    dict(heads=3), dict(heads=0), dict(heads=70000), dict(row_blocks=1 << 28), dict(requests=1 << 31),
                    dict(tokens=1 << 31), dict(most=0), dict(starts=None), dict(starts=None, tokens=3),
                    dict(starts=None, most=1), dict(requests=60000, row_blocks=1 << 26)):
            assert call(some, at, C.byref(_window(**bad)), None) == ARG, bad
        for bad in (dict(k_token=-128), dict(k_token=1 << 26), dict(v_token=-128), dict(v_token=1 << 26)):
            assert call(some, C.byref(cache(**bad)), C.byref(_window()), None) == ARG, bad
        for bad in (dict(q=AT + 4), dict(q_token=4), dict(q_head=1), dict(out=AT + 8), dict(out_token=2), dict(out_head=12)):
            assert call(some, at, C.byref(_window(**bad)), None) == ALIGN, bad
        assert call(some, at, C.byref(_window(requests=0, q=None)), None) == 0
        assert call(some, at, C.byref(_window(tokens=0, q=None)), None) == 0
    assert lib.pgcm_kv_window_reserve(None, 4, 2, 128, None) == ARG
    for bad in ((4, 3, 128), (0, 1, 128), (4, 2, 12), (4, 2, 264)):
        assert lib.pgcm_kv_window_reserve(some, *bad, None) == ARG, bad


def test_tensors_on_the_host_are_refused():
    with pytest.raises(ValueError, match="CUDA"):
        pgcm.KV8Cache(*ref.pool8(1, 2, 16, 2, 64, torch.int8))
    with pytest.raises(ValueError, match="8 bits"):
        pgcm.KV8Cache(torch.zeros(2, 16, 2, 64, dtype=torch.uint8), None, None, None)
    x = torch.zeros(1, 2, 64)
    with pytest.raises(ValueError, match="CUDA"):
        pgcm.kv8_append(None, None, x, x, None, None, None)
    for move in (pgcm.kv8_store, pgcm.kv8_load):
        with pytest.raises(ValueError, match="CUDA"):
            move(None, None, torch.zeros(1, dtype=torch.int32))
    for call in (pgcm.kv8_attend, pgcm.kv_window):
        with pytest.raises(ValueError, match="CUDA"):
            call(None, x, None, None, None)


@pytest.mark.parametrize("code", ref.CODES)
def test_the_reference_rounds_as_torch_does(code):
    """the definitions' codes against torch's conversion, over all sizes"""
    x = torch.from_numpy(__import__("numpy").random.default_rng(5).standard_normal(4096)) * 2.0 ** torch.randint(-16, 6, (4096,))
    x = x[x.abs() <= ref.TOP[code]].float()
    got = ref.rounded(x.double().numpy(), code)
    want = x.round() if code == torch.int8 else x.to(code).float()
    assert torch.equal(torch.from_numpy(got).float(), want)
