"""pgcm_kv_append and pgcm_kv_summarize against their definitions."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2411_03357_amd as pgcm

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def _table(positions, dim):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2).double() / dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _near(got, want, x, half, dim, what):
    """rounded once to half; before that dim + 8 roundings of 2^-24 of the size of the rotated pair"""
    size = want.abs().nan_to_num().amax(-1, keepdim=True)
    tol = ref.UNIT[half] * 1.001 * want.abs().nan_to_num() + ref.LEAST[half] + (dim + 8) * 2.0 ** -23 * size
    nans = want.isnan()
    got = got.double().cpu()
    assert torch.equal(got.isnan(), nans), what
    assert bool(((got - want).abs().nan_to_num() <= tol).all()), what


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("dim,rope_dim,adjacent", [(128, 128, False), (128, 128, True), (64, 64, False), (80, 80, True),
                                                   (80, 48, False), (256, 256, False), (256, 64, True), (96, 96, False),
                                                   (8, 0, False), (24, 16, False), (128, 0, True)])
def test_append(half, dim, rope_dim, adjacent):
    for tokens, heads, kv, normed in ((1, 1, 1, (True, True)), (7, 6, 2, (True, False)), (33, 40, 40, (False, True)),
                                      (3, 5, 1, (False, False))):
        block, blocks = 16, 9
        rng = np.random.default_rng([dim, tokens])
        x = ref.numbers(dim + tokens, tokens, heads + 2 * kv, dim).to(half)
        weights = [(1 + ref.numbers(i, dim, std=0.3)).to(half) if n else None for i, n in enumerate(normed)]
        positions = rng.integers(0, 50, tokens)
        table = _table(50, rope_dim) if rope_dim else None
        slots = rng.permutation(block * blocks)[:tokens]
        packed = x.cuda()
        q, k, v = packed[:, :heads], packed[:, heads:heads + kv], packed[:, heads + kv:]
        pool = torch.full((blocks, 2, block, kv, dim), 7.0, dtype=half, device="cuda")
        out = torch.empty(tokens, heads, dim, dtype=half, device="cuda")
        pgcm.kv_append(pgcm.KVCache(pool[:, 0], pool[:, 1]), q, k, v,
                       torch.from_numpy(positions.astype(np.int32)).cuda() if rope_dim else None,
                       torch.from_numpy(slots.astype(np.int64)).cuda(), out,
                       q_weight=None if weights[0] is None else weights[0].cuda(),
                       k_weight=None if weights[1] is None else weights[1].cuda(), eps=1e-5,
                       rope=None if table is None else table.cuda(), adjacent=adjacent)
        want = [ref.turned(x[:, a:b], w, 1e-5, table, positions, adjacent)
                for a, b, w in ((0, heads, weights[0]), (heads, heads + kv, weights[1]))]
        _near(out, want[0], x[:, :heads], half, dim, "q")
        pool = pool.cpu()
        at = (slots // block, slots % block)
        _near(pool[:, 0][at], want[1], x[:, heads:heads + kv], half, dim, "k")
        assert torch.equal(pool[:, 1][at], x[:, heads + kv:])
        pool[:, 0][at] = 7.0
        pool[:, 1][at] = 7.0
        assert bool((pool == 7.0).all())        # nothing else was written


@pytest.mark.parametrize("tokens,heads,kv,dim", [(4097, 3, 1, 64), (2100, 8, 2, 128), (4100, 20, 10, 80), (1400, 16, 8, 256)])
def test_append_many_tokens(tokens, heads, kv, dim):
    """workgroups of one wavefront to four"""
    half, block = BF16, 32
    blocks = -(-tokens // block)
    x = ref.numbers(6, tokens, heads + 2 * kv, dim).to(half)
    weight, table = (1 + ref.numbers(7, dim, std=0.3)).to(half), _table(tokens, dim)
    slots = np.random.default_rng(8).permutation(block * blocks)[:tokens]
    packed, pool = x.cuda(), torch.empty(blocks, 2, block, kv, dim, dtype=half, device="cuda")
    out = torch.empty(tokens, heads, dim, dtype=half, device="cuda")
    pgcm.kv_append(pgcm.KVCache(pool[:, 0], pool[:, 1]), packed[:, :heads], packed[:, heads:heads + kv], packed[:, heads + kv:],
                   torch.arange(tokens, dtype=torch.int32).cuda(), torch.from_numpy(slots).cuda(), out,
                   q_weight=weight.cuda(), k_weight=weight.cuda(), eps=1e-5, rope=table.cuda())
    want = ref.turned(x[:, :heads + kv], weight, 1e-5, table, range(tokens), False)
    _near(out, want[:, :heads], None, half, dim, "q")
    at, pool = (slots // block, slots % block), pool.cpu()
    _near(pool[:, 0][at], want[:, heads:], None, half, dim, "k")
    assert torch.equal(pool[:, 1][at], x[:, heads + kv:])


def test_append_passes_over_slots_and_marks_positions():
    half, kv, dim = BF16, 2, 64
    x = ref.numbers(3, 6, 4 + 2 * kv, dim).to(half)
    packed = x.cuda()
    pool = torch.full((2, 2, 16, kv, dim), 7.0, dtype=half, device="cuda")
    slots = torch.tensor([-1, 0, 32, 31, 1 << 40, 5]).cuda()
    positions = torch.tensor([0, 9, 1, -1, 2, 10], dtype=torch.int32).cuda()
    table = _table(10, dim)
    # in place: q_out is q
    pgcm.kv_append(pgcm.KVCache(pool[:, 0], pool[:, 1]), packed[:, :4], packed[:, 4:4 + kv], packed[:, 4 + kv:], positions,
                   slots, packed[:, :4], rope=table.cuda())
    want_q = ref.turned(x[:, :4], None, 0, table, positions.tolist(), False)
    want_k = ref.turned(x[:, 4:4 + kv], None, 0, table, positions.tolist(), False)
    _near(packed[:, :4], want_q, x[:, :4], half, dim, "q")
    flat = pool.transpose(1, 2).reshape(32, 2, kv, dim).cpu()
    for t, slot in enumerate(slots.tolist()):
        if 0 <= slot < 32:
            _near(flat[slot, 0], want_k[t], None, half, dim, "k")
            assert torch.equal(flat[slot, 1], x[t, 4 + kv:])
            flat[slot] = 7.0
    assert bool((flat == 7.0).all())


def test_append_keys_alone_into_another_order():
    half, kv, dim = F16, 3, 128
    x = ref.numbers(4, 5, 2 * kv, dim).to(half)
    k, v = torch.zeros(kv, 4, 32, dim, dtype=half, device="cuda"), torch.zeros(4, kv, 32, dim, dtype=half, device="cuda")
    packed = x.cuda()
    pgcm.kv_append(pgcm.KVCache(k.permute(1, 2, 0, 3), v.permute(0, 2, 1, 3)), None, packed[:, :kv], packed[:, kv:], None,
                   torch.tensor([0, 33, 66, 127, 64]).cuda(), None)
    for t, (b, i) in enumerate(((0, 0), (1, 1), (2, 2), (3, 31), (2, 0))):
        assert torch.equal(k[:, b, i].cpu(), x[t, :kv]) and torch.equal(v[b, :, i].cpu(), x[t, kv:])


def test_append_beyond_4_GiB():
    kv, dim, block = 8, 128, 16
    blocks = (1 << 32) // (block * kv * dim) + 3
    k = torch.empty(blocks, block, kv, dim, dtype=F16, device="cuda")
    k[0], k[-1] = 0, 0
    x = ref.numbers(5, 2, kv, dim).to(F16).cuda()
    pgcm.kv_append(pgcm.KVCache(k, k), None, x, x, None, torch.tensor([blocks * block - 1, 3]).cuda(), None)
    assert torch.equal(k[-1, -1], x[0]) and torch.equal(k[0, 3], x[1])
    assert int((k[-1] != 0).any(-1).sum()) == kv and int((k[0] != 0).any(-1).sum()) == kv


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("dim,block,kv", [(128, 16, 2), (64, 32, 3), (80, 48, 1), (256, 16, 2), (8, 16, 1), (136, 64, 5)])
def test_summarize(half, dim, block, kv):
    n = 11
    k = ref.numbers(dim + block, n, block, kv, dim).to(half)
    k[2, 1, 0, 3], k[3, 0, 0, 0], k[4, 2, 0, 1] = math.nan, math.inf, -math.inf
    k[5] = 0
    k[6] *= 1e-4
    counts = [block, 1, 2, 5, block, block, block, 0, -3, block + 7, 15]
    rng = np.random.default_rng(dim)
    blocks, entries = rng.permutation(n), rng.permutation(n + 5)[:n]
    where = torch.empty_like(k)
    where[blocks] = k
    bounds = torch.full((n + 5, kv, 2, dim), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((n + 5, kv), 99.0, device="cuda")
    pgcm.kv_summarize(pgcm.KVCache(where.cuda(), where.cuda()), torch.from_numpy(blocks.astype(np.int32)).cuda(),
                      torch.tensor(counts, dtype=torch.int32).cuda(), bounds, scales,
                      entries=torch.from_numpy(entries.astype(np.int32)).cuda())
    want = ref.summarize(k, counts)
    bounds, scales = bounds.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(bounds[entries], want[0]) and np.array_equal(scales[entries], want[1])
    rest = np.setdiff1d(np.arange(n + 5), entries)
    assert (bounds[rest] == 99).all() and (scales[rest] == 99).all()
    # entries default to the blocks' numbers; what lies outside is passed over
    bounds = torch.full((n, kv, 2, dim), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((n, kv), 99.0, device="cuda")
    pgcm.kv_summarize(pgcm.KVCache(where.cuda(), where.cuda()), torch.tensor([4, -1, n, 1 << 30], dtype=torch.int32).cuda(),
                      torch.full((4,), block, dtype=torch.int32).cuda(), bounds, scales)
    want = ref.summarize(where[4:5], [block])
    assert np.array_equal(bounds[4:5].cpu().numpy(), want[0]) and np.array_equal(scales[4:5].cpu().numpy(), want[1])
    assert int((bounds != 99).flatten(1).any(1).sum()) <= 1 and int((scales != 99).any(1).sum()) == 1


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dim,rope_dim", [(128, 0), (128, 128), (128, 64), (80, 48), (256, 32), (24, 16)])
def test_append_infinities_and_nan(half, adjacent, dim, rope_dim):
    """channels that are not rotated stay as they are beside any others, and a pair that is rotated sees its own two alone"""
    tokens, heads, kv = 5, 4, 2
    x = ref.numbers(dim + rope_dim, tokens, heads + 2 * kv, dim).to(half)
    x[0, :, dim - 1], x[1, :, dim - 2], x[2, :, dim - 3] = math.inf, -math.inf, math.nan
    x[3, :, 1], x[4, :, 2] = math.nan, math.inf
    packed = x.cuda()
    pool = torch.zeros(2, 2, 16, kv, dim, dtype=half, device="cuda")
    out = torch.empty(tokens, heads, dim, dtype=half, device="cuda")
    positions, slots = [3, 9, 1, 7, 8], [0, 17, 3, 31, 5]
    table = _table(10, rope_dim) if rope_dim else None
    pgcm.kv_append(pgcm.KVCache(pool[:, 0], pool[:, 1]), packed[:, :heads], packed[:, heads:heads + kv], packed[:, heads + kv:],
                   torch.tensor(positions, dtype=torch.int32).cuda() if rope_dim else None, torch.tensor(slots).cuda(), out,
                   rope=None if table is None else table.cuda(), adjacent=adjacent)
    rows = pool.transpose(1, 2).reshape(32, 2, kv, dim).cpu()[slots]
    want = ref.turned(x[:, :heads + kv], None, 0, table, positions, adjacent)
    got = torch.cat([out.cpu(), rows[:, 0]], 1)
    still = x[:, :heads + kv, rope_dim:]
    assert torch.equal(got[..., rope_dim:].isnan(), still.isnan())
    assert torch.equal(got[..., rope_dim:].nan_to_num(7.0), still.nan_to_num(7.0))
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    there = want.isfinite()
    _near(got.where(there, 0.0), want.where(there, 0.0), None, half, dim, "q and k")
    assert torch.equal(rows[:, 1].nan_to_num(7.0), x[:, heads + kv:].nan_to_num(7.0))


def test_append_a_table_without_lines():
    """... is no table that can be left out"""
    x = torch.ones(2, 4, 64, dtype=F16, device="cuda")
    pool = torch.zeros(2, 2, 16, 2, 64, dtype=F16, device="cuda")
    at = torch.zeros(2, dtype=torch.int32, device="cuda")
    for shape in ((0, 64), (5, 0)):
        with pytest.raises(pgcm.PgcmError) as e:
            pgcm.kv_append(pgcm.KVCache(pool[:, 0], pool[:, 1]), None, x[:, :2], x[:, 2:], at, torch.tensor([1, 2]).cuda(), None,
                           rope=torch.empty(shape, device="cuda"))
        assert e.value.status == -1


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dim,rope_dim", [(128, 0), (128, 48), (80, 16)])
def test_append_copies_what_is_neither_normed_nor_rotated(half, adjacent, dim, rope_dim):
    """numbers below the normal ones, infinities; without rotation to the last bit, zeros of both signs among them"""
    bits = np.random.default_rng(dim).integers(-(1 << 15), 1 << 15, (9, 6, dim)).astype(np.int16)
    bits[:, :, -1], bits[:, :, -2], bits[:, :, -3] = -32768, 0, 1
    x = torch.from_numpy(bits).view(half)
    x[x.isnan()] = -0.0
    packed = x.cuda()
    pool = torch.zeros(1, 2, 16, 2, dim, dtype=half, device="cuda")
    out = torch.empty(9, 2, dim, dtype=half, device="cuda")
    at = torch.zeros(9, dtype=torch.int32).cuda() if rope_dim else None
    pgcm.kv_append(pgcm.KVCache(pool[:, 0], pool[:, 1]), packed[:, :2], packed[:, 2:4], packed[:, 4:], at,
                   torch.arange(9).cuda(), out, rope=_table(3, rope_dim).cuda() if rope_dim else None, adjacent=adjacent)
    for got, want in ((out, x[:, :2]), (pool[0, 0, :9], x[:, 2:4]), (pool[0, 1, :9], x[:, 4:])):
        got, want = [x[..., rope_dim:].cpu().contiguous() for x in (got, want)]
        assert torch.equal(got, want) and (rope_dim != 0 or torch.equal(got.view(torch.int16), want.view(torch.int16)))
