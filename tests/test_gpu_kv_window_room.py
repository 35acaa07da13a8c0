"""Attention with a window: what a workspace takes from the device."""
import pytest
import torch

import paper_2411_03357_amd as pgcm

pytestmark = pytest.mark.gpu

MIB = 1 << 20


def _taken(space, new, kv, heads, length, dim=128, block=16):
    """bytes of the device that are gone after a call"""
    pool = torch.zeros(length // block, 2, block, kv, dim, dtype=torch.bfloat16, device="cuda")
    cache = pgcm.KVCache(pool[:, 0], pool[:, 1])
    q = torch.zeros(new, heads, dim, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    tables = torch.arange(length // block, dtype=torch.int32, device="cuda")[None]
    lens, starts = [torch.tensor(x, dtype=torch.int32).cuda() for x in ([length], [0, new])]
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    pgcm.kv_window(cache, q, tables, lens, out, starts=starts, most=new, workspace=space)
    torch.cuda.synchronize()
    return before - torch.cuda.mem_get_info()[0]


def test_a_call_takes_room_for_its_own_parts():
    """of 8 new tokens, 4 heads to a kv head: an item of each kv head, each part 128 rows of 130 floats; rules give no item more than
    one part for 8 tiles of 64 tokens.  A workspace grows by half as much again, and allocations are of whole 2 MiB"""
    for kv, length in ((1, 2048), (8, 16384)):
        _taken(pgcm.KVWorkspace(), 8, kv, 4 * kv, length)       # (the code is on the device)
        parts = kv * length // 64 // 8
        taken = _taken(pgcm.KVWorkspace(), 8, kv, 4 * kv, length)
        assert taken <= 1.5 * parts * 128 * 130 * 4 + 4 * MIB, (kv, length, taken)


def test_after_a_reservation_calls_take_nothing():
    space = pgcm.KVWorkspace()
    pgcm.kv_window_reserve(space, 64, 8, 128)
    for new, kv, heads, length in ((1, 8, 64, 65536), (8, 1, 16, 65536), (100, 8, 64, 32768), (8, 8, 32, 65536)):
        _taken(pgcm.KVWorkspace(), new, kv, heads, length)
        assert _taken(space, new, kv, heads, length) == 0
