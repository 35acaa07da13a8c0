"""pgcm_kv_attend against its definition in 64 bits: lengths from none to several tiles of several workgroups, blocks that
are not there, whatever the pool holds elsewhere, orders of memory, groups of heads, selections, weights, graphs, streams."""
import copy
import math
import threading

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2411_03357_amd as pgcm

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def _run(r, q, scale=None, selected=None, kept=None, decay=1.0, weigh=False, **more):
    n, heads, dim = q.shape
    cache = pgcm.KVCache(*r.on_gpu())
    tables, lens = r.gpu_tables()
    out = torch.full((n, heads, dim), 9.0, dtype=r.half, device="cuda")
    lse = torch.full((n, heads), 9.0, device="cuda")
    weights = torch.full((n, r.most), 9.0, device="cuda") if weigh else None
    sel = None if selected is None else torch.from_numpy(np.ascontiguousarray(selected, dtype=np.int32)).cuda()
    for _ in range(2):      # twice: what workgroups count each other by must be left clean
        pgcm.kv_attend(cache, q.cuda(), tables, lens, out, lse=lse, scale=scale, selected=sel, weights=weights,
                       kept=None if kept is None else kept.cuda(), decay=decay, **more)
    return out, lse, weights


def _check(r, q, scale=None, selected=None, kept=None, decay=1.0, weigh=False, **more):
    """... and again with room for more tokens in the tables, which is worked on in another way"""
    _check_once(r, q, scale, selected, kept, decay, weigh, **more)
    wide = copy.copy(r)
    wide.most += -(-2200 // r.block)
    wide.tables = np.pad(r.tables, ((0, 0), (0, wide.most - r.most)), constant_values=-1)
    if selected is not None:
        selected = np.pad(selected, ((0, 0), (0, 0), (0, wide.most - r.most)), constant_values=-1)
    if kept is not None:
        kept = torch.nn.functional.pad(kept, (0, wide.most - r.most))
    _check_once(wide, q, scale, selected, kept, decay, weigh, **more)


def _check_once(r, q, scale, selected, kept, decay, weigh, **more):
    out, lse, weights = _run(r, q, scale, selected, kept, decay, weigh, **more)
    want = ref.attend(r, q, r.dim ** -0.5 if scale is None else scale, selected, kept, decay)
    ref.within(out, want[0], "out")
    ref.within(lse, want[1], "lse")
    if weigh:
        ref.within(weights, want[2], "weights")


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("dim", [8, 64, 72, 80, 128, 136, 256])
def test_lengths(half, dim):
    r = ref.Requests(dim, [1, 0, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300], 2, dim, half)
    _check(r, ref.numbers(dim, 12, 4, dim, std=2.0).to(half))


@pytest.mark.parametrize("kv,group", [(1, 1), (3, 1), (1, 5), (2, 16), (1, 17), (1, 40), (2, 33)])
def test_heads(kv, group):
    r = ref.Requests(kv * 100 + group, [70, 0, 261], kv, 128, F16)
    _check(r, ref.numbers(group, 3, kv * group, 128, std=2.0).to(F16))


@pytest.mark.parametrize("block", [16, 32, 48, 256])
@pytest.mark.parametrize("junk", [math.nan, math.inf, -65504.0])
def test_blocks_that_are_not_there(block, junk):
    """holes in every row; a row of nothing but holes; numbers beyond the pool; junk wherever no token is"""
    r = ref.Requests(block, [400, 33, 150, 90, 1], 2, 64, F16, block=block, holes=0.4, junk=junk)
    r.tables[3, :] = -1
    r.tables[2, 0] = r.blocks           # not a block of the pool
    r.tables[1, 0] = 0x7FFFFFFF
    kept = ref.numbers(5, 5, r.most).float().abs()
    _check(r, ref.numbers(block, 5, 4, 64).to(F16), kept=kept, decay=0.75, weigh=True)


def test_lengths_beyond_the_row_and_below_zero():
    r = ref.Requests(9, [64, 64, 64], 1, 64, BF16)
    q = ref.numbers(9, 3, 2, 64).to(BF16)
    cache = pgcm.KVCache(*r.on_gpu())
    tables = torch.from_numpy(r.tables[:, :4].copy()).cuda()
    out, lse = torch.empty(3, 2, 64, dtype=BF16, device="cuda"), torch.empty(3, 2, device="cuda")
    pgcm.kv_attend(cache, q.cuda(), tables, torch.tensor([1 << 30, -5, 64], dtype=torch.int32).cuda(), out, lse=lse)
    want = ref.attend(r, q, 64 ** -0.5)
    ref.within(out[::2], (want[0][0][::2], want[0][1][::2]), "out")
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())


def test_no_requests_and_rows_without_blocks():
    r = ref.Requests(10, [20], 1, 64, BF16)
    cache = pgcm.KVCache(*r.on_gpu())
    none = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    pgcm.kv_attend(cache, none, torch.empty(0, 3, dtype=torch.int32, device="cuda"),
                   torch.empty(0, dtype=torch.int32, device="cuda"), none)
    q = torch.ones(2, 2, 64, dtype=BF16, device="cuda")
    pgcm.kv_attend(cache, q, torch.empty(2, 0, dtype=torch.int32, device="cuda"),
                   torch.tensor([5, 0], dtype=torch.int32).cuda(), q, weights=torch.empty(2, 0, device="cuda"))
    assert bool((q == 0).all())


@pytest.mark.parametrize("order", ["btkd", "bktd", "kbtd", "tbkd"])
def test_orders_of_memory_and_strides(order):
    r = ref.Requests(11, [100, 47], 3, 80, F16, order=order)
    q = ref.numbers(11, 2, 6, 80).to(F16)
    k, v = r.on_gpu()
    wide = torch.full((2, 3, 6, 96), math.nan, dtype=F16, device="cuda")
    wide[:, 1, :, :80] = q.cuda()
    out = torch.full((2, 6, 2, 80), 3.0, dtype=F16, device="cuda")
    tables = torch.full((2, 2 * r.most + 1), -7, dtype=torch.int32, device="cuda")
    tables[:, 1:r.most + 1] = torch.from_numpy(r.tables).cuda()
    pgcm.kv_attend(pgcm.KVCache(k, v), wide[:, 1, :, :80], tables[:, 1:r.most + 1], r.gpu_tables()[1], out[:, :, 1])
    ref.within(out[:, :, 1], ref.attend(r, q, 80 ** -0.5)[0], "out")
    assert bool((out[:, :, 0] == 3.0).all())


@pytest.mark.parametrize("dim,kv,group", [(128, 1, 8), (64, 2, 1), (256, 1, 3)])
def test_one_request_in_many_workgroups(dim, kv, group):
    r = ref.Requests(dim, [20011], kv, dim, BF16)
    q = ref.numbers(dim, 1, kv * group, dim, std=3.0).to(BF16)
    out, lse, _ = _run(r, q)
    # (the reference takes a long row as one)
    k = r.k[r.tables[0, :-1]].flatten(0, 1)[:20011].double()
    v = r.v[r.tables[0, :-1]].flatten(0, 1)[:20011].double()
    s = torch.einsum("hgd,nhd->hgn", q[0].double().view(kv, group, dim), k) * dim ** -0.5
    top = torch.logsumexp(s, -1)
    p = (s - top[..., None]).exp()
    want = torch.einsum("hgn,nhd->hgd", p, v).reshape(1, kv * group, dim)
    e = (dim + 2) * 2.0 ** -24 * dim ** -0.5 * \
        float(torch.einsum("hgd,nhd->hgn", q[0].double().view(kv, group, dim).abs(), k.abs()).max())
    off = 2 * e + 20027 * 2.0 ** -24 + 2.0 ** -22 * (1.5 * float(s.abs().max()) + 4)
    size = torch.einsum("hgn,nhd->hgd", p, v.abs()).reshape(1, kv * group, dim)
    ref.within(out, (want, ref.UNIT[BF16] * want.abs() + (off + 2.0 ** -16) * 1.01 * size), "out")
    ref.within(lse, (top.reshape(1, -1), torch.full_like(top.reshape(1, -1), off)), "lse")
    again, lse2, _ = _run(r, q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dim,group,tokens", [(64, 1, 9000), (128, 16, 7001), (128, 3, 13000), (256, 20, 5000)])
def test_parts_joined_in_groups(dim, group, tokens):
    r = ref.Requests(21, [tokens, 40], 1, dim, BF16, holes=0.2)
    _check(r, ref.numbers(21, 2, group, dim).to(BF16), weigh=True)


def test_many_requests():
    """more than the lanes of a wavefront, most of them short or empty, as one batch"""
    rng = np.random.default_rng(5)
    lens = [int(v) for v in rng.choice([0, 0, 1, 5, 16, 40, 130], 150)]
    lens[:70] = [0] * 70
    r = ref.Requests(12, lens, 1, 64, BF16)
    kept = ref.numbers(6, 150, r.most).float()
    _check(r, ref.numbers(12, 150, 2, 64).to(BF16), kept=kept, decay=0.5, weigh=True)


def test_large_scores_and_scales():
    r = ref.Requests(13, [200, 60], 1, 128, BF16)
    q = ref.numbers(13, 2, 3, 128, std=30.0).to(BF16)
    for scale in (0.0, -0.02, 0.2):
        _check(r, q, scale=scale)


@pytest.mark.parametrize("half", [F16, BF16])
def test_small_weights_beside_a_large_one(half):
    """a first token that has nearly all of the weight and no value, and many whose weights are 2^-20.6 of its: what is left
    of these in halves must be as exact as the output.  Three hundred requests that share their blocks, so that a wavefront
    takes many tokens of one."""
    r = ref.Requests(15, [2048], 1, 64, half)
    r.v = r.v.abs()
    r.k[:, :, :, 0] = -14.296875
    r.k[int(r.tables[0, 0]), 0], r.v[int(r.tables[0, 0]), 0] = 0, 0
    q = torch.zeros(1, 2, 64, dtype=half)
    q[:, :, 0] = 1
    want = ref.attend(r, q, 1.0)
    r.tables, r.lens = np.repeat(r.tables, 300, 0), r.lens * 300
    out, lse, _ = _run(r, q.expand(300, 2, 64).contiguous(), scale=1.0)
    ref.within(out, [x.expand(300, 2, 64) for x in want[0]], "out")
    ref.within(lse, [x.expand(300, 2) for x in want[1]], "lse")


def test_nan_of_a_request_stays_its_own():
    r = ref.Requests(14, [40, 40], 1, 64, BF16)
    q = ref.numbers(14, 2, 2, 64).to(BF16)
    q[0, 0, 3] = math.nan
    out, lse, _ = _run(r, q)
    assert bool(out[0, 0].isnan().all()) and bool(lse[0, 0].isnan())
    assert bool(out[0, 1].isfinite().all()) and bool(out[1].isfinite().all())


@pytest.mark.parametrize("keep", [1, 3, 9, 40])
def test_selected_blocks(keep):
    """lists that end in -1, name places beyond the request, in any order, and blocks that are not there"""
    rng = np.random.default_rng(keep)
    r = ref.Requests(15, [400, 16, 0, 333], 2, 64, F16, holes=0.2)
    selected = np.full((4, 2, keep), -1)
    for b in range(4):
        for g in range(2):
            at = rng.permutation(r.most + 2)[:keep]
            selected[b, g, :at.size] = at
    selected[0, 0, 0] = 1 << 30
    _check(r, ref.numbers(15, 4, 10, 64).to(F16), selected=selected)


def test_selected_matches_all():
    r = ref.Requests(16, [500, 77], 2, 128, F16)
    q = ref.numbers(16, 2, 8, 128).to(F16)
    every = np.broadcast_to(np.arange(r.most), (2, 2, r.most))
    _check(r, q, selected=every)


def test_weights_in_place():
    r = ref.Requests(17, [100, 31], 2, 64, F16)
    q = ref.numbers(17, 2, 4, 64).to(F16)
    kept = ref.numbers(18, 2, r.most).float().abs()
    weights = kept.cuda()
    pgcm.kv_attend(pgcm.KVCache(*r.on_gpu()), q.cuda(), *r.gpu_tables(), torch.empty_like(q, device="cuda"), weights=weights,
                   kept=weights, decay=0.25)
    ref.within(weights, ref.attend(r, q, 0.125, None, kept, 0.25)[2], "weights")


def test_a_pool_of_more_than_4_GiB():
    """elements beyond 2^32 of the pool; a block's values lie just before its keys"""
    kv, dim, block = 8, 128, 16
    blocks = (1 << 32) // (block * kv * dim) + 40
    pool = torch.empty(blocks, block, kv, dim, dtype=F16, device="cuda")
    r = ref.Requests(19, [block * 3 + 5], kv, dim, F16)
    at = [blocks - 1, 1, blocks - 20, blocks // 2]
    k, v = r.on_gpu()
    for j, b in enumerate(at):
        pool[b].copy_(k[int(r.tables[0, j])])
        pool[b - 1].copy_(v[int(r.tables[0, j])])
    tables = torch.tensor([at], dtype=torch.int32).cuda() - 1
    q = ref.numbers(19, 1, kv, dim).to(F16)
    out = torch.empty(1, kv, dim, dtype=F16, device="cuda")
    pgcm.kv_attend(pgcm.KVCache(pool[1:], pool[:-1]), q.cuda(), tables, r.gpu_tables()[1], out)
    ref.within(out, ref.attend(r, q, dim ** -0.5)[0], "out")


def test_captured_into_a_graph():
    """lengths and contents change between replays; other calls of the workspace come in between"""
    r = ref.Requests(20, [700, 5000, 20], 2, 128, BF16)
    q = ref.numbers(20, 3, 8, 128).to(BF16)
    cache = pgcm.KVCache(*r.on_gpu())
    tables, lens = r.gpu_tables()
    dq, out = q.cuda(), torch.empty_like(q, device="cuda")
    kept, weights = torch.rand(3, r.most, device="cuda"), torch.empty(3, r.most, device="cuda")
    space = pgcm.KVWorkspace()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(pgcm.PgcmError) as e:
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
                torch.zeros(4, device="cuda")
                pgcm.kv_attend(cache, dq, tables, lens, out, weights=weights, kept=kept, workspace=space)
        assert e.value.status == -7         # a captured call does not allocate
        space.reserve(3, 8, 2, 128, 16, r.most)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            pgcm.kv_attend(cache, dq, tables, lens, out, weights=weights, kept=kept, workspace=space)
        for step in range(4):
            now = [[700, 5000, 20], [0, 4999, 3], [1, 1, 1], [690, 130, 17]][step]
            lens.copy_(torch.tensor(now, dtype=torch.int32))
            dq.mul_(-0.9)
            graph.replay()
            got, got_weights = out.clone(), weights.clone()
            pgcm.kv_attend(cache, dq, tables, lens, out, weights=weights, kept=kept, workspace=space)
            torch.cuda.synchronize()
            assert torch.equal(got, out) and torch.equal(got_weights, weights)
            if step == 1:       # grows the workspace: the graph keeps what it was captured with
                space.reserve(300, 8, 2, 128, 16, r.most)
    space.destroy()


def test_another_stream_and_threads():
    import threading
    r = ref.Requests(21, [3000, 40], 2, 128, BF16)
    q = ref.numbers(21, 2, 4, 128).to(BF16)
    cache = pgcm.KVCache(*r.on_gpu())
    tables, lens = r.gpu_tables()
    want, _, _ = _run(r, q)
    dq = q.cuda()
    torch.cuda.synchronize()
    wrong = []

    def work():
        stream = torch.cuda.Stream()
        out = torch.empty_like(dq)
        for _ in range(20):
            pgcm.kv_attend(cache, dq, tables, lens, out, stream=stream)
        stream.synchronize()
        if not torch.equal(out, want):
            wrong.append(1)
    threads = [threading.Thread(target=work) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_threads_on_one_stream():
    """calls of several launches and of growing sizes, on the stream's own workspace"""
    jobs = []
    for n, tokens in enumerate((300, 900, 2500, 6000)):
        r = ref.Requests(30 + n, [tokens, 50], 2, 64, BF16)
        cache, q = pgcm.KVCache(*r.on_gpu()), ref.numbers(30 + n, 2, 8, 64).to(BF16).cuda()
        tables, lens = r.gpu_tables()
        jobs.append((cache, q, tables, lens, torch.zeros_like(q), torch.zeros(2, r.most, device="cuda")))
    want = []
    for cache, q, tables, lens, out, weights in jobs:
        pgcm.kv_attend(cache, q, tables, lens, out, weights=weights)
        want.append((out.clone(), weights.clone()))
    torch.cuda.synchronize()
    wrong = []

    def work(job, expected):
        cache, q, tables, lens, out, weights = job
        for _ in range(200):
            pgcm.kv_attend(cache, q, tables, lens, out, weights=weights)
            if not (torch.equal(out, expected[0]) and torch.equal(weights, expected[1])):
                wrong.append(q.shape)

    threads = [threading.Thread(target=work, args=x) for x in zip(jobs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_weights_count_in_32_bits(half, dim):
    """values that cancel, channel by channel for one head each, so that what weights are off by is what is left.  Four tokens
    with scores up to 1 and four with scores of 0, whose values make up the others' sum: of a first four channels a head, of
    sixteen.  One channel of the keys counts, so that a score is off by 2^-23 of itself and the exponential's argument by as
    much again; a weight by these, its exponential (2^-23) and what halves leave of it (binary16: 2^-22); then eight
    additions, the total's eight and its reciprocal (2^-24 each)."""
    heads, n, block = 16, 4, 16
    rng = np.random.default_rng(31)
    s = torch.from_numpy(rng.uniform(0.5, 1, n)).to(half).double()
    f = torch.from_numpy(rng.uniform(0.5, 1, heads)).to(half).double()
    v = torch.from_numpy(rng.standard_normal((2 * n, dim))).to(half).double()
    w = torch.cat([(f[:, None] * s).exp(), torch.ones(heads, n, dtype=torch.float64)], 1)
    for h in range(heads):
        for c in range(4 * h, 4 * h + 4):
            left = -(w[h, :n] @ v[:n, c])
            for i in range(n, 2 * n):
                v[i, c] = left.to(half).double()
                left = left - v[i, c]
    w = w / w.sum(1, keepdim=True)
    want, size = w @ v, w @ v.abs()
    off = (4 * float(f.max() * s.max()) + 2 + 2 + 9) * 2.0 ** -23
    tol = ref.UNIT[half] * want.abs() + ref.LEAST[half] + 1.01 * off * size
    k_cache = torch.zeros(1, block, 1, dim, dtype=half)
    v_cache = torch.zeros_like(k_cache)
    k_cache[0, :n, 0, 5], v_cache[0, :2 * n, 0] = s.to(half), v.to(half)
    q = torch.zeros(1, heads, dim, dtype=half)
    q[0, :, 5] = f.to(half)
    for row in (1, 200):        # a workgroup for the item; tables with room for many tiles
        tables = torch.zeros(1, row, dtype=torch.int32).cuda()
        out = torch.empty_like(q, device="cuda")
        pgcm.kv_attend(pgcm.KVCache(k_cache.cuda(), v_cache.cuda()), q.cuda(), tables,
                       torch.tensor([2 * n], dtype=torch.int32).cuda(), out, scale=1.0)
        ref.within(out[0], (want, tol), "out")


@pytest.mark.parametrize("half", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_infinities_and_nan_that_are_attended_to(half, dim):
    """a value that is infinite makes its channel infinite, one that is no number makes it none, and no other channel, head or
    request sees it; alone in a request, whose weight is exactly 1, among others, and in several parts of a long one"""
    r = ref.Requests(22, [1, 17, 300, 2500, 40], 2, dim, half)
    at = lambda b, t: (int(r.tables[b, t // 16]), t % 16)
    for b, t in ((0, 0), (1, 16), (2, 40), (2, 299), (3, 5), (3, 2499)):
        i, inside = at(b, t)
        r.v[i, inside, 0, 3], r.v[i, inside, 0, dim - 1] = math.inf, -math.inf
        r.v[i, inside, 1, 6] = math.nan
    i, inside = at(3, 1300)
    r.v[i, inside, 0, 3] = -math.inf        # of both signs in one channel: no number
    q = ref.numbers(22, 5, 6, dim).to(half)
    (want, tol), _, _ = ref.attend(r, q, dim ** -0.5)
    assert bool(want[:3, :3, 3].isposinf().all()) and bool(want[:4, :3, dim - 1].isneginf().all())
    assert bool(want[3, :3, 3].isnan().all()) and bool(want[:4, 3:, 6].isnan().all())
    assert int((~want.isfinite()).sum()) == 4 * 3 * 3
    for row in (r.most, r.most + 2200 // 16):
        wide = copy.copy(r)
        wide.tables, wide.most = np.pad(r.tables, ((0, 0), (0, row - r.most)), constant_values=-1), row
        out = _run(wide, q)[0].double().cpu()
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.isposinf(), want.isposinf())
        assert torch.equal(out.isneginf(), want.isneginf())
        there = want.isfinite()
        assert bool(((out - want).abs()[there] <= tol[there]).all())


@pytest.mark.parametrize("row", [4, 300])
def test_selections_without_places(row):
    """... are selections: nothing is attended to; and, like others, they go with no weights"""
    q = torch.ones(2, 4, 64, dtype=F16, device="cuda")
    pool = torch.ones(8, 16, 2, 64, dtype=F16, device="cuda")
    tables = torch.zeros(2, row, dtype=torch.int32, device="cuda")
    lens = torch.tensor([40, 0], dtype=torch.int32, device="cuda")
    none = torch.empty(2, 2, 0, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 9.0), torch.full((2, 4), 9.0, device="cuda")
    pgcm.kv_attend(pgcm.KVCache(pool, pool), q, tables, lens, out, lse=lse, selected=none)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    with pytest.raises(pgcm.PgcmError) as e:
        pgcm.kv_attend(pgcm.KVCache(pool, pool), q, tables, lens, out, selected=none, weights=torch.zeros(2, row, device="cuda"))
    assert e.value.status == -1


def _attend_on_gpu(pool, tables, lens, q, scale, heads_of):
    """out, lse, weights in 64 bits of long requests, on the device, and how far each may be off: as in kv_reference, but for
    the additions, of which a token passes through less than 1024, as wavefronts of 256 workgroups share a request's tokens"""
    n, heads, dim = q.shape
    blocks, _, block, kv, _ = pool.shape
    f = torch.float64
    out, lse = torch.zeros(n, heads, dim, dtype=f, device="cuda"), torch.full((n, heads), -math.inf, dtype=f, device="cuda")
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    weights = torch.zeros(tables.shape, dtype=f, device="cuda")
    weights_tol = torch.zeros_like(weights)
    unit = ref.UNIT[pool.dtype]
    for b, t in enumerate(lens):
        place = torch.arange(-(-t // block), device="cuda")
        place = place[tables[b, :place.numel()] >= 0]
        token = (place[:, None] * block + torch.arange(block, device="cuda")).flatten()
        there = token < t
        if not bool(there.any()):
            continue
        at = tables[b, place].long()
        for g in range(kv):
            k, v = [pool[at, i, :, g].flatten(0, 1)[there].to(f) for i in (0, 1)]
            mine = slice(g * heads_of, (g + 1) * heads_of)
            x = q[b, mine].to(f)
            s = (x @ k.T) * scale
            e = (dim + 2) * 2.0 ** -24 * scale * (x.abs() @ k.abs().T).amax(1)
            off = 2 * e + 1040 * 2.0 ** -24 + 2.0 ** -22 * (s.abs().amax(1) * 1.5 + 4)
            lse[b, mine], lse_tol[b, mine] = torch.logsumexp(s, 1), off
            p = (s - lse[b, mine, None]).exp()
            out[b, mine] = p @ v
            out_tol[b, mine] = unit * out[b, mine].abs() + ref.LEAST[pool.dtype] + (off + 2.0 ** -22)[:, None] * 1.01 * (p @ v.abs())
            where = token[there] // block
            weights[b].index_add_(0, where, p.sum(0))
            weights_tol[b].index_add_(0, where, ((off + heads * 2.0 ** -24)[:, None] * p).sum(0))
    return (out, out_tol), (lse, lse_tol), (weights, weights_tol)


@pytest.mark.parametrize("dim,kv,group,half,lens", [
    # spans of 36 tiles and more, over requests of all lengths: more than a segment each
    (64, 4, 5, F16, [0, 150001, 5, 70007, 0, 33333, 16, 1, 46000, 129, 8000, 0]),
    (128, 2, 8, BF16, [300000, 0, 17, 129, 200003, 60000, 0, 1, 4095]),
    # 256 channels, a workgroup a compute unit: short spans, and long ones
    (256, 2, 3, BF16, [90000, 40, 0, 30011, 128, 7, 2000]),
    (256, 2, 17, F16, [200003, 0, 1000, 90001, 64]),
])
def test_long_requests_of_all_lengths(dim, kv, group, half, lens):
    block = 32
    gen = torch.Generator(device="cuda").manual_seed(dim + group)
    most = max(-(-t // block) for t in lens) + 1
    here = torch.zeros(len(lens), most, dtype=torch.bool)
    for b, t in enumerate(lens):
        here[b, :-(-t // block)] = True
    here = here.cuda() & (torch.rand(here.shape, device="cuda", generator=gen) >= 0.05)
    n = int(here.sum())
    tables = torch.full(here.shape, -1, dtype=torch.int32, device="cuda")
    tables[here] = torch.randperm(n + 3, device="cuda", generator=gen)[:n].to(torch.int32)
    pool = torch.empty(n + 3, 2, block, kv, dim, dtype=half, device="cuda").normal_(generator=gen)
    for b, t in enumerate(lens):        # what lies beyond a request is no number
        j = t // block
        if t % block and int(tables[b, j]) >= 0:
            pool[int(tables[b, j]), :, t % block:] = math.nan
    q = torch.empty(len(lens), kv * group, dim, dtype=half, device="cuda").normal_(0, 2.5, generator=gen)
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
    weights = torch.full(tables.shape, 9.0, device="cuda")
    cache, d_lens = pgcm.KVCache(pool[:, 0], pool[:, 1]), torch.tensor(lens, dtype=torch.int32).cuda()
    pgcm.kv_attend(cache, q, tables, d_lens, out, lse=lse, weights=weights)
    want = _attend_on_gpu(pool, tables, lens, q, dim ** -0.5, group)
    for got, (value, tol), what in zip((out, lse, weights), want, ("out", "lse", "weights")):
        ref.within(got, (value.cpu(), tol.cpu()), what)
    again, alone = torch.empty_like(out), torch.empty_like(out)
    pgcm.kv_attend(cache, q, tables, d_lens, again)
    assert torch.equal(out, again)          # without weights, and to the last bit
    for b in (1, len(lens) - 2):            # a request by itself, cut in other places
        pgcm.kv_attend(cache, q[b:b + 1], tables[b:b + 1], d_lens[b:b + 1], alone[b:b + 1])
        ref.within(alone[b], (want[0][0][b].cpu(), want[0][1][b].cpu()), "alone")


@pytest.mark.parametrize("half", [F16, BF16])
def test_scores_that_are_not_finite(half):
    """minus infinity has no weight, and of a whole request gives none; what is plus infinity or no number spoils its head alone"""
    r = ref.Requests(23, [40, 40, 2100], 1, 64, half)
    q = ref.numbers(23, 3, 3, 64).to(half)
    q[:, 0, 7], q[:, 1, 7], q[:, 2, 7] = 1, -1, 0.5
    q[1, 2, 7] = 1
    r.k[int(r.tables[0, 1]), 3, 0, 7] = math.inf
    r.k[int(r.tables[2, 70]), 3, 0, 7] = -math.inf
    for j in range(3):
        r.k[int(r.tables[1, j]), :, 0, 7] = -math.inf
    for row in (r.most, r.most + 200):
        wide = copy.copy(r)
        wide.tables, wide.most = np.pad(r.tables, ((0, 0), (0, row - r.most)), constant_values=-1), row
        out, lse, _ = _run(wide, q)
        bad = torch.tensor([[True, False, True], [False, True, False], [False, True, False]])
        assert torch.equal(lse.isnan().cpu(), bad) and torch.equal(out.isnan().all(-1).cpu(), bad)
        assert torch.equal(out.isnan().any(-1).cpu(), bad)
        assert bool((lse[1, ::2] == -math.inf).all()) and bool((out[1, ::2] == 0).all())
        for b, h, j in ((0, 1, 1), (2, 0, 70), (2, 2, 70)):     # the others: as if that token were not there
            less = copy.copy(r)
            less.k = r.k.clone()
            less.k[int(r.tables[b, j]), 3, 0] = 0
            want = ref.attend(less, q, 0.125)
            p0 = (0.0 - want[1][0][b, h]).exp()                 # ... whose score of 0 is taken out again
            v0 = r.v[int(r.tables[b, j]), 3, 0].double()
            out_h = (want[0][0][b, h] - p0 * v0) / (1 - p0)
            tol = (want[0][1][b, h] + ref.UNIT[half] * out_h.abs()) / (1 - p0)
            ref.within(out[b, h], (out_h, tol), "out")


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_large_finite_values(dim):
    """... whose products with a query leave the range of binary32: they are looked at again, and count as they are"""
    r = ref.Requests(24, [300, 1, 40], 2, dim, BF16)
    r.v, r.k = r.v * 2.0 ** 80, r.k * 2.0 ** -60
    q = (ref.numbers(24, 3, 6, dim) * 2.0 ** 60).to(BF16)
    _check(r, q)
