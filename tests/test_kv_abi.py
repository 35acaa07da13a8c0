"""The C ABI of the operators on KV blocks: exported, and arguments refused before anything reaches the GPU."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import paper_2411_03357_amd as pgcm
from paper_2411_03357_amd import kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, ALIGN = -1, -2
AT = 1 << 20            # an address; no call here gets as far as using it


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "pgcm_kv.h")).read()
    names = sorted(set(re.findall(r"\b(pgcm_kv_[a-z_0-9]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(pgcm.KV_EXPORTS) == names and len(names) == 8
    lib = C.CDLL(pgcm.library_path())
    for n in names:
        assert hasattr(lib, n), n


def test_importing_the_package_does_not_import_torch():
    import subprocess
    import sys
    code = "import sys, paper_2411_03357_amd; sys.exit('torch' in sys.modules)"
    assert subprocess.run([sys.executable, "-c", code], cwd=ROOT).returncode == 0
    with pytest.raises(AttributeError):
        pgcm.no_such_name


def _cache(**change):
    c = kv._Cache(AT, AT, 0, 10, 16, 2, 128, 0, 8192, 256, 128, 8192, 256, 128)
    for name, value in change.items():
        setattr(c, name, value)
    return c


BAD_CACHES = [dict(k=None), dict(v=None), dict(half=2), dict(reserved=1), dict(blocks=0), dict(blocks=1 << 31),
              dict(block_tokens=0), dict(block_tokens=8), dict(block_tokens=24), dict(block_tokens=4112), dict(kv_heads=0),
              dict(kv_heads=70000), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264)]
UNALIGNED_CACHES = [dict(k=AT + 8), dict(v=AT + 2), dict(k_block=4), dict(k_token=129), dict(k_head=-4), dict(v_block=1),
                    dict(v_token=12), dict(v_head=2)]


def _attend(**change):
    a = kv._Attend(3, 4, AT, 512, 128, AT, 20, 20, 0.1, AT, None, 0, 1.0, AT, 512, 128, None, None, None)
    for name, value in change.items():
        setattr(a, name, value)
    return a


def _append(**change):
    a = kv._Append(5, 4, AT, AT, AT, 512, 128, 256, 128, 256, 128, AT, AT, AT, AT, 1e-6, 0, AT, 100, 128, AT, 512, 128)
    for name, value in change.items():
        setattr(a, name, value)
    return a


def _select(**change):
    a = kv._Select(3, 4, 2, 128, 1, 16, AT, 512, 128, AT, 20, 20, 50, AT, AT, AT, 5, 1, 1, AT, None)
    for name, value in change.items():
        setattr(a, name, value)
    return a


def _evict(**change):
    a = kv._Evict(3, 20, 16, 50, AT, AT, 20, AT, AT, 4, 1, 1, AT, AT, AT, 20)
    for name, value in change.items():
        setattr(a, name, value)
    return a


def test_caches_are_refused():
    lib, some = kv._lib(), C.create_string_buffer(256)
    for bad, status in [(b, ARG) for b in BAD_CACHES] + [(b, ALIGN) for b in UNALIGNED_CACHES]:
        cache = _cache(**bad)
        at = C.addressof(cache)
        assert lib.pgcm_kv_attend(some, at, C.byref(_attend()), None) == status, bad
        assert lib.pgcm_kv_append(at, C.byref(_append()), None) == status, bad
        assert lib.pgcm_kv_summarize(at, 3, AT, AT, None, 10, AT, AT, None) == status, bad


def test_attend_refuses():
    lib, some, cache = kv._lib(), C.create_string_buffer(256), _cache()
    at = C.addressof(cache)
    assert lib.pgcm_kv_attend(None, at, C.byref(_attend()), None) == ARG
    assert lib.pgcm_kv_attend(some, None, C.byref(_attend()), None) == ARG
    assert lib.pgcm_kv_attend(some, at, None, None) == ARG
    for bad in (dict(q=None), dict(out=None), dict(lens=None), dict(tables=None), dict(scale=math.nan),
                dict(scale=math.inf), dict(heads=3), dict(heads=0), dict(heads=70000), dict(requests=70000),
                dict(row_blocks=1 << 28), dict(selected=AT, keep=2, weights=AT), dict(kept=AT),
                dict(requests=60000, row_blocks=1 << 26)):
        assert lib.pgcm_kv_attend(some, at, C.byref(_attend(**bad)), None) == ARG, bad
    for bad in (dict(k_token=-128), dict(k_token=1 << 26), dict(v_token=-128), dict(v_token=1 << 26)):
        other = _cache(**bad)
        assert lib.pgcm_kv_attend(some, C.byref(other), C.byref(_attend()), None) == ARG, bad
    for bad in (dict(q=AT + 4), dict(q_request=4), dict(q_head=1), dict(out=AT + 8), dict(out_request=2), dict(out_head=12)):
        assert lib.pgcm_kv_attend(some, at, C.byref(_attend(**bad)), None) == ALIGN, bad
    assert lib.pgcm_kv_attend(some, at, C.byref(_attend(requests=0, q=None)), None) == 0


def test_append_refuses():
    lib, cache = kv._lib(), _cache()
    at = C.addressof(cache)
    assert lib.pgcm_kv_append(at, None, None) == ARG and lib.pgcm_kv_append(None, C.byref(_append()), None) == ARG
    for bad in (dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None),
                dict(heads=3), dict(heads=0), dict(heads=70000), dict(eps=-1.0), dict(eps=math.nan), dict(rope_dim=0),
                dict(rope_dim=24), dict(rope_dim=144), dict(rope_positions=0), dict(tokens=1 << 31)):
        assert lib.pgcm_kv_append(at, C.byref(_append(**bad)), None) == ARG, bad
    for bad in (dict(q=AT + 2), dict(k=AT + 2), dict(v=AT + 2), dict(q_out=AT + 2), dict(q_token=3), dict(q_head=3),
                dict(k_token=3), dict(k_head=3), dict(v_token=3), dict(v_head=3), dict(q_out_token=3), dict(q_out_head=3),
                dict(q_weight=AT + 2), dict(k_weight=AT + 2), dict(rope=AT + 4)):
        assert lib.pgcm_kv_append(at, C.byref(_append(**bad)), None) == ALIGN, bad
    assert lib.pgcm_kv_append(at, C.byref(_append(tokens=0, k=None)), None) == 0


def test_summarize_refuses():
    lib, cache = kv._lib(), _cache()
    at = C.addressof(cache)
    good = [at, 3, AT, AT, None, 10, AT, AT, None]
    for i, value, status in ((0, None, ARG), (1, 1 << 31, ARG), (2, None, ARG), (3, None, ARG), (5, 0, ARG), (5, 1 << 31, ARG),
                             (6, None, ARG), (7, None, ARG), (6, AT + 8, ALIGN)):
        args = list(good)
        args[i] = value
        assert lib.pgcm_kv_summarize(*args) == status, (i, value)
    good[1] = 0
    assert lib.pgcm_kv_summarize(*good) == 0


def test_select_refuses():
    lib, some = kv._lib(), C.create_string_buffer(256)
    assert lib.pgcm_kv_select(None, C.byref(_select()), None) == ARG and lib.pgcm_kv_select(some, None, None) == ARG
    for bad in (dict(half=2), dict(heads=3), dict(heads=0), dict(kv_heads=0), dict(head_dim=20), dict(head_dim=264),
                dict(block_tokens=20), dict(q=None), dict(tables=None), dict(lens=None), dict(bounds=None), dict(scales=None),
                dict(selected=None), dict(keep=0), dict(entry_count=0), dict(entry_count=1 << 31), dict(requests=70000),
                dict(row_blocks=1 << 28)):
        assert lib.pgcm_kv_select(some, C.byref(_select(**bad)), None) == ARG, bad
    for bad in (dict(q=AT + 2), dict(q_request=3), dict(q_head=3), dict(bounds=AT + 8)):
        assert lib.pgcm_kv_select(some, C.byref(_select(**bad)), None) == ALIGN, bad
    assert lib.pgcm_kv_select(some, C.byref(_select(requests=0, q=None)), None) == 0


def test_evict_refuses():
    lib = kv._lib()
    assert lib.pgcm_kv_evict(None, None) == ARG
    for bad in (dict(block_tokens=0), dict(block_tokens=20), dict(row_blocks=1 << 28), dict(blocks=1 << 31), dict(most=1 << 31),
                dict(requests=1 << 31), dict(weights=None), dict(tables=None), dict(lens=None), dict(evict=None),
                dict(victims=None)):
        assert lib.pgcm_kv_evict(C.byref(_evict(**bad)), None) == ARG, bad
    assert lib.pgcm_kv_evict(C.byref(_evict(requests=0, lens=None)), None) == 0


def test_workspace_refuses():
    lib, some = kv._lib(), C.create_string_buffer(256)
    assert lib.pgcm_kv_create(None) == ARG
    lib.pgcm_kv_destroy(None)
    assert lib.pgcm_kv_reserve(None, 1, 4, 2, 128, 16, 10, None) == ARG
    for bad in ((1, 3, 2, 128, 16, 10), (1, 0, 2, 128, 16, 10), (1, 4, 0, 128, 16, 10), (1, 4, 2, 100, 16, 10),
                (1, 4, 2, 128, 20, 10), (1, 4, 2, 128, 16, 1 << 28)):
        assert lib.pgcm_kv_reserve(some, *bad, None) == ARG, bad


def test_the_binding_checks_tensors():
    k = torch.zeros(4, 16, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="CUDA"):
        pgcm.KVCache(k, k)
    with pytest.raises(ValueError, match="float16"):
        pgcm.KVCache(k.float(), k.float())
    with pytest.raises(ValueError, match="must be"):
        pgcm.KVCache(k, k[:2])
    w = torch.zeros(2, 5)
    with pytest.raises(ValueError):
        pgcm.kv_evict(w, torch.zeros(2, 5, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), 16, w, w)
    with pytest.raises(ValueError):
        pgcm.kv_select(w, torch.zeros(2, dtype=torch.int32), w, w, w, 16, w)


def test_what_no_launch_holds_is_refused():
    """2^32 threads or more"""
    lib, some, cache, one = kv._lib(), C.create_string_buffer(256), _cache(), _cache(kv_heads=1, head_dim=8)
    for tokens in (1 << 26, (1 << 31) - 1):
        assert lib.pgcm_kv_append(C.addressof(cache), C.byref(_append(tokens=tokens)), None) == ARG
    for c, n in ((cache, 1 << 25), (cache, 1 << 30), (one, (1 << 31) - 1)):
        assert lib.pgcm_kv_summarize(C.addressof(c), n, AT, AT, None, 10, AT, AT, None) == ARG
    wide = dict(heads=1024, kv_heads=1024, row_blocks=1)
    assert lib.pgcm_kv_select(some, C.byref(_select(requests=1 << 14, **wide)), None) == ARG
    assert lib.pgcm_kv_select(some, C.byref(_select(requests=65535, **wide)), None) == ARG
    for n, row in ((1 << 24, 1), ((1 << 31) - 1, 20), (1 << 24, 2048), (1 << 22, 2049)):
        assert lib.pgcm_kv_evict(C.byref(_evict(requests=n, row_blocks=row)), None) == ARG
