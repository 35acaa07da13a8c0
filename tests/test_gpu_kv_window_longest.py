"""Attention with a window over requests of about as many tokens as a call holds: rows of a table that name one block over and over."""
import math

import pytest
import torch

import paper_2411_03357_amd as pgcm

pytestmark = pytest.mark.gpu

BLOCK = 4096


@pytest.mark.parametrize("length", [1 << 29, (1 << 30) - 5, (1 << 31) - BLOCK])
@pytest.mark.parametrize("new", [1, 2])
def test_every_part_of_the_longest_requests_counts(length, new):
    """one block weighs more than all others together, wherever it lies"""
    dim, places = 64, -(-length // BLOCK)
    k, v = [torch.zeros(2, BLOCK, 1, dim, dtype=torch.float16, device="cuda") for _ in "kv"]
    k[1, :, 0, 0], v[0], v[1] = 1.0, 1.0, 2.0
    q = torch.zeros(new, 1, dim, dtype=torch.float16, device="cuda")
    q[:, 0, 0] = 64.0
    cache = pgcm.KVCache(k, v)
    lens, starts = [torch.tensor(x, dtype=torch.int32).cuda() for x in ([length], [0, new])]
    for at in (0, 1, places // 3, places // 2, places - 300, places - 2):
        tables = torch.zeros(1, places, dtype=torch.int32, device="cuda")
        tables[0, at] = 1
        out, lse = torch.zeros_like(q), torch.zeros(new, 1, device="cuda")
        pgcm.kv_window(cache, q, tables, lens, out, lse=lse, scale=1.0, starts=starts, most=new)
        # of the weights, 2^31 / (4096 e^64) < 2^-73 are not that block's
        assert bool((out == 2).all()), (at, out.unique().tolist())
        want = 64 + math.log(BLOCK)
        assert bool(((lse.double() - want).abs() <= 2.0 ** -20 * want).all()), (at, lse.tolist())
