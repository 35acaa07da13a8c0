"""What is built with torch and what without, and for which torch."""
import sys
import types

import pytest
import torch

import paper_2411_03357_amd as pgcm
from paper_2411_03357_amd import build, kv


def test_the_cipher_is_built_without_torch(monkeypatch):
    made = []
    monkeypatch.setattr(build, "_host_build", lambda source, target, *more: made.append(source))
    build.build_marshal()
    assert made == ["marshal.cpp", "kv_marshal.cpp"]
    del made[:]
    monkeypatch.setitem(sys.modules, "torch", None)      # an import of it fails
    build.build_marshal()
    assert made == ["marshal.cpp"]


def test_stale_without_and_for_another_torch(monkeypatch, tmp_path):
    for name in ("LIB", "MARSHAL", "KV_MARSHAL"):
        at = tmp_path / name
        at.write_bytes(b"..." + build._built_for(torch) + b"...")
        monkeypatch.setattr(build, name, str(at))
    assert not build.is_stale()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", torch.__version__ + "1")
        assert build.is_stale()
    (tmp_path / "KV_MARSHAL").unlink()
    assert build.is_stale()
    monkeypatch.setitem(sys.modules, "torch", None)
    assert not build.is_stale()


def test_an_extension_of_another_torch_is_refused(monkeypatch):
    kv._load_marshal()
    monkeypatch.setitem(sys.modules, "paper_2411_03357_amd._kv_marshal", None)
    monkeypatch.delattr(pgcm, "_kv_marshal", raising=False)
    with pytest.raises(ImportError, match="not built"):
        kv._load_marshal()
    other = types.SimpleNamespace(built_for="built for torch 0.1")
    monkeypatch.setattr(pgcm, "_kv_marshal", other, raising=False)
    with pytest.raises(ImportError, match="built for torch 0.1, and this is torch"):
        kv._load_marshal()
