"""Which workspace calls get that name none: one for each stream."""
import gc
import threading

import pytest

from paper_2411_03357_amd import kv


class _Space:
    alive = 0

    def __init__(self):
        _Space.alive += 1

    def __del__(self):
        _Space.alive -= 1


@pytest.fixture
def spaces(monkeypatch):
    monkeypatch.setattr(kv, "KVWorkspace", _Space)
    monkeypatch.setattr(kv, "_workspaces", {})
    monkeypatch.setattr(kv, "_device", lambda: 0)


def _in_threads(n, stream):
    got, together = [], threading.Barrier(n)

    def work():
        a = kv.kv_workspace(stream)
        assert kv.kv_workspace(stream) is a
        got.append(id(a))
        together.wait()     # all of them at once
    threads = [threading.Thread(target=work) for _ in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return got


def test_a_stream_has_one_workspace_in_all_threads(spaces):
    assert len(set(_in_threads(4, 1 << 20))) == 1
    assert kv.kv_workspace(1 << 20) is not kv.kv_workspace(1 << 21)
    assert kv.kv_workspace(0) is kv.kv_workspace(0)


def test_the_stream_of_each_thread_has_one_of_its_own(spaces):
    """hipStreamPerThread is one handle for another stream in each thread"""
    assert len(set(_in_threads(4, 2))) == 4
    gc.collect()
    assert _Space.alive == 0            # they end with their threads
