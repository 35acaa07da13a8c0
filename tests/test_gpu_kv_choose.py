"""pgcm_kv_select and pgcm_kv_evict against their definitions: whole numbers, so exactly."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2411_03357_amd as pgcm

pytestmark = pytest.mark.gpu


def _select(seed, lens, kv, group, dim, keep, first, last, half=torch.bfloat16, block=16, most=None, coarse=False, odd=None):
    rng = np.random.default_rng([80, seed])
    n = len(lens)
    most = most or max(1, max(-(-t // block) for t in lens)) + 2
    entries = max(4, most * 2)
    tables = rng.integers(0, entries, (n, most)).astype(np.int32)
    tables[rng.random((n, most)) < 0.1] = -1
    tables[0, :2] = entries, 0x7FFFFFFF
    ends = rng.integers(-2, 3, (entries, kv, 2, dim)) if coarse else rng.integers(-127, 128, (entries, kv, 2, dim))
    bounds = np.sort(ends, axis=2).astype(np.int8)
    scales = (np.full((entries, kv), 0.25) if coarse else rng.random((entries, kv))).astype(np.float32)
    if coarse:
        bounds[:] = bounds[:1]          # all the same: the first ones win
        scales[entries // 2:] = 0.0
    q = ref.numbers(seed, n, kv * group, dim).to(half)
    if odd is not None:
        odd(q, scales)
    want = ref.select(q, tables, lens, bounds.astype(np.int64), scales, block, keep, first, last)
    selected = torch.full((n, kv, keep), 55, dtype=torch.int32, device="cuda")
    counts = torch.full((n, kv), 55, dtype=torch.int32, device="cuda")
    for _ in range(2):
        pgcm.kv_select(q.cuda(), torch.from_numpy(tables).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                       torch.from_numpy(bounds).cuda(), torch.from_numpy(scales).cuda(), block, selected, counts, first=first,
                       last=last)
    assert np.array_equal(selected.cpu().numpy(), want)
    assert np.array_equal(counts.cpu().numpy(), (want >= 0).sum(-1))


@pytest.mark.parametrize("half", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [8, 64, 72, 128, 136, 256])
def test_select(half, dim):
    _select(dim, [0, 1, 16, 17, 333, 2000, -4], 2, 3, dim, 7, 1, 2, half)


@pytest.mark.parametrize("kv,group", [(1, 1), (3, 16), (1, 17), (2, 40)])
def test_select_heads(kv, group):
    _select(group, [900, 64], kv, group, 64, 9, 0, 1)


@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 1, 1), (5, 3, 4), (3, 100, 0), (40, 2, 2), (500, 0, 1),
                                             (7, 0, 4000000000)])
def test_select_ends(keep, first, last):
    _select(keep, [600, 90, 16, 0], 2, 2, 64, keep, first, last, block=32)


@pytest.mark.parametrize("keep", [1, 9, 64])
def test_select_equal_scores(keep):
    _select(keep, [1600, 200], 1, 2, 64, keep, 0, 0, coarse=True)


@pytest.mark.parametrize("blocks,keep", [(511, 20), (513, 200), (5000, 300), (20000, 1000)])
def test_select_long_rows(blocks, keep):
    """a row in several workgroups; one too long for a workgroup's memory"""
    _select(blocks, [16 * blocks - 3, 100], 1, 2, 64, keep, 1, 1)


def test_select_what_is_not_a_number():
    def odd(q, scales):
        q[0, 0, :3] = torch.tensor([math.nan, math.inf, -math.inf])
        q[0, 1] = 0
        q[1, 2] = 1e-38
        scales[::3] = 1e30
    _select(3, [700, 500], 2, 2, 64, 11, 1, 1, odd=odd)


def test_select_many_requests():
    rng = np.random.default_rng(8)
    _select(4, [int(v) for v in rng.integers(0, 400, 90)], 2, 2, 64, 6, 1, 1)


# ---------------------------------------------------------------------------------------------
def _evict(seed, lens, asked, most, first, last, block=16, row=None, weights=None, blocks=1000, in_place=False):
    rng = np.random.default_rng([81, seed])
    n = len(lens)
    row = row or max(1, max(-(-t // block) for t in lens)) + 2
    if weights is None:
        weights = np.exp(rng.standard_normal((n, row)) * 3)
    weights = weights.astype(np.float32)
    wide = rng.integers(0, blocks, (n, row + 3)).astype(np.int32)
    wide[rng.random(wide.shape) < 0.2] = -1
    wide[0, 1] = blocks
    tables = wide[:, 1:row + 1]
    want = ref.evict(weights, tables, lens, block, asked, most, first, last, blocks)
    d_wide = torch.from_numpy(wide).cuda()
    d_tables = d_wide[:, 1:row + 1]
    out = d_tables if in_place else torch.full((n, row), 55, dtype=torch.int32, device="cuda")
    victims = torch.full((n, most), 55, dtype=torch.int32, device="cuda")
    victim_blocks = torch.full((n, most), 55, dtype=torch.int32, device="cuda")
    pgcm.kv_evict(torch.from_numpy(weights).cuda(), d_tables, torch.tensor(lens, dtype=torch.int32).cuda(), block,
                  torch.tensor(asked, dtype=torch.int32).cuda(), victims, victim_blocks, out, first=first, last=last,
                  blocks=blocks)
    assert np.array_equal(victims.cpu().numpy(), want)
    left = tables.copy()
    want_blocks = np.full((n, most), -1)
    for b in range(n):
        at = want[b][want[b] >= 0]
        want_blocks[b, :at.size] = tables[b, at]
        left[b, at] = -1
    assert np.array_equal(victim_blocks.cpu().numpy(), want_blocks)
    assert np.array_equal(out.cpu().numpy(), left)
    wide[:, 1:row + 1] = left if in_place else tables
    assert np.array_equal(d_wide.cpu().numpy(), wide)


@pytest.mark.parametrize("first,last", [(0, 0), (1, 2), (5, 0), (0, 9), (4000000000, 1), (1, 4000000000)])
def test_evict(first, last):
    _evict(first % 100 + last % 100, [0, 1, 16, 17, 300, 5000, -9, 1000], [3, 1, 2, 2, 5, 64, 4, 0], 64, first, last)


@pytest.mark.parametrize("row", [16384, 16390, 20000])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_long_rows(row, in_place):
    _evict(row, [16 * row, 16 * row - 5000], [700, 3], 700, 1, 0, row=row, in_place=in_place)


def test_evict_equal_and_odd_weights():
    n, row = 4, 70
    weights = np.ones((n, row))
    weights[1, ::2] = -0.0
    weights[1, 1::2] = 0.0
    weights[2] = np.resize([math.nan, math.inf, -math.inf, 1e-45, 3.4e38, -1.0], row)
    weights[3] = math.nan
    for asked in (1, 10, 33, 70):
        _evict(asked, [16 * row] * n, [asked] * n, 70, 0, 0, row=row, weights=weights, in_place=True)


def test_evict_beyond_what_there_is():
    _evict(6, [100, 100, 1 << 30], [1 << 30, -1, 7], 50, 0, 1, row=9)


def test_evict_nothing_asked_for():
    w = torch.ones(2, 5, device="cuda")
    tables = torch.arange(10, dtype=torch.int32).view(2, 5).cuda()
    lens = torch.tensor([80, 80], dtype=torch.int32).cuda()
    victims = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(tables)
    pgcm.kv_evict(w, tables, lens, 16, lens, victims, None, out)
    assert torch.equal(out, tables)
    pgcm.kv_evict(w[:0], tables[:0], lens[:0], 16, lens[:0], victims[:0])


@pytest.mark.parametrize("dim,half", [(64, torch.bfloat16), (80, torch.float16), (256, torch.bfloat16)])
def test_select_rows_of_a_workgroup_each(dim, half):
    """as many lists as compute units, with room for 385 to 1024 blocks"""
    rng = np.random.default_rng(dim)
    lens = [int(v) for v in rng.integers(0, 16 * 300, 32)]
    lens[3], lens[7], lens[11] = 16 * 1000 - 1, 0, 16 * 700
    _select(dim + 1, lens, 8, 2, dim, 40, 1, 2, half, most=(1000, 385, 1024)[dim % 3])


@pytest.mark.parametrize("dim,group", [(72, 5), (80, 17), (128, 2), (136, 1), (256, 3)])
@pytest.mark.parametrize("lens,keep", [([16 * 599, 100], 30), ([16 * 5000 - 3, 0, 40, 16 * 700], 300), ([16 * 8190], 7)])
def test_select_rows_in_parts(dim, group, lens, keep):
    """scored by many workgroups, sixteen blocks a wavefront or four times as many, before the choice"""
    _select(dim + keep, lens, 2 if keep != 300 else 4, group, dim, keep, 1, 1, torch.float16 if dim == 80 else torch.bfloat16)
