"""Attention with a window, over blocks in 8 bits and of halves, against its definition in 64 bits."""
import math

import pytest
import torch

import paper_2411_03357_amd as pgcm
import kv8_reference as ref8
import kv_reference as ref16
import kv_window_reference as ref

pytestmark = pytest.mark.gpu

HALVES = [torch.float16, torch.bfloat16]
KINDS = [(h, c) for h in HALVES for c in (None,) + ref8.CODES]
NAMES = ["%s-%s" % (str(h)[6:], "halves" if c is None else str(c)[6:]) for h, c in KINDS]
kinds = pytest.mark.parametrize("kind", KINDS, ids=NAMES)


def _blocks(kind, seed, lens, kv, dim, **more):
    half, code = kind
    return ref.Blocks(seed, lens, kv, dim, half, **more) if code is None else ref.Blocks8(seed, lens, kv, dim, half, code, **more)


def _q(seed, rows, heads, dim, half, std=1.0):
    return ref16.numbers(seed, rows, heads, dim, std=std).to(half)


@kinds
@pytest.mark.parametrize("window, sinks", [(0, 0), (1, 0), (5, 1), (16, 16), (17, 4), (100, 40), (129, 0), (5000, 3)])
def test_single_tokens(kind, window, sinks):
    lens = [0, 1, 15, 16, 17, 31, 33, 64, 129, 260, 513, 1000]
    b = _blocks(kind, 1, lens, 2, 128)
    ref.check(pgcm, b, _q(2, len(lens), 8, 128, kind[0], 2.0), [1] * len(lens), window, sinks)


@kinds
@pytest.mark.parametrize("kv, group, dim, block", [(1, 1, 16, 16), (3, 5, 64, 32), (2, 16, 80, 48), (2, 17, 128, 64), (1, 40, 256, 16),
                                                   (5, 3, 144, 16), (40, 1, 128, 16), (1, 2, 48, 4096)])
def test_heads_and_sizes(kind, kv, group, dim, block):
    lens = [70, 3, 200, 0, 129]
    for seed, (window, sinks) in enumerate([(0, 0), (50, 20)]):
        b = _blocks(kind, 3 + seed, lens, kv, dim, block=block)
        ref.check(pgcm, b, _q(4, len(lens), kv * group, dim, kind[0]), [1] * len(lens), window, sinks)


@pytest.mark.parametrize("half", HALVES)
def test_eight_channels_of_halves(half):
    for dim in (8, 24, 120):
        b = _blocks((half, None), 8, [70, 3, 200], 2, dim)
        ref.check(pgcm, b, _q(4, 3, 4, dim, half), [1] * 3, 50, 20)


@kinds
def test_holes(kind):
    lens = [40, 300, 700, 16]
    for seed, holes, window, sinks in ((5, 0.4, 0, 0), (6, 0.7, 200, 40), (7, 1.0, 0, 0), (7, 1.0, 30, 4)):
        b = _blocks(kind, seed, lens, 2, 128, holes=holes)
        ref.check(pgcm, b, _q(6, len(lens), 4, 128, kind[0]), [1] * len(lens), window, sinks)


@kinds
@pytest.mark.parametrize("lens, kv, group, dim, window, sinks", [
    ([20011, 3, 7000, 0, 12345], 2, 4, 128, 0, 0), ([20011, 3, 7000, 0, 12345], 2, 4, 128, 6000, 100),
    ([70001], 1, 2, 64, 0, 0), ([40000], 1, 16, 128, 0, 0), ([9000, 5000], 1, 8, 256, 0, 3), ([3000] * 3, 3, 20, 80, 2500, 64)])
def test_long_ones_in_parts(kind, lens, kv, group, dim, window, sinks):
    b = _blocks(kind, 9, lens, kv, dim)
    ref.check(pgcm, b, _q(10, len(lens), kv * group, dim, kind[0]), [1] * len(lens), window, sinks)


@kinds
@pytest.mark.parametrize("rows, most, kv, group, dim, window, sinks, holes", [
    (80, 700, 4, 2, 64, 0, 0, 0.1), (16, 1000, 16, 3, 128, 200, 20, 0.0), (40, 400, 4, 17, 128, 0, 0, 0.2), (33, 500, 8, 1, 80, 300, 7, 0.3),
    (65, 600, 4, 5, 256, 0, 0, 0.0), (32, 3000, 8, 8, 144, 2500, 64, 0.1), (128, 300, 4, 16, 24, 0, 3, 0.0)])
def test_heads_side_by_side(kind, rows, most, kv, group, dim, window, sinks, holes):
    """four heads a workgroup, items cut into few parts; lengths of all sizes"""
    lens = [(most - 1) * (7 * i % rows) // (rows - 1) for i in range(rows)]
    b = _blocks(kind, 51, lens, kv, dim, holes=holes)
    q = _q(52, rows, kv * group, dim, kind[0])
    if kind[1] is not None and dim % 16:   # (rows of codes are whole sixteens of bytes)
        with pytest.raises(pgcm.PgcmError):
            ref.run(pgcm, b, q, [1] * rows, window, sinks)
        return
    first = ref.check(pgcm, b, q, [1] * rows, window, sinks)
    for _ in range(2):
        again = ref.run(pgcm, b, q, [1] * rows, window, sinks)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


@kinds
def test_heads_side_by_side_in_many_parts(kind):
    """parts joined in two steps: an item's, alone, and beside items without tokens"""
    for lens in ([140000], [140000, 0, 5]):
        b = _blocks(kind, 53, lens, 16, 16)
        ref.check(pgcm, b, _q(54, len(lens), 48, 16, kind[0]), [1] * len(lens))


@pytest.mark.parametrize("kind", [x for x in KINDS if x[1] is not None], ids=[n for x, n in zip(KINDS, NAMES) if x[1] is not None])
def test_heads_side_by_side_of_new_tokens(kind):
    lens, news = [900, 30, 0, 5, 300], [60, 33, 3, 10, 16]
    b = _blocks(kind, 55, lens, 4, 128)
    ref.check(pgcm, b, _q(56, sum(news), 8, 128, kind[0]), news, 0, 0, spare=4, most=60)


@kinds
def test_heads_side_by_side_in_a_graph(kind):
    """replayed with other lengths, between eager calls of one head a workgroup on its workspace"""
    rows, most = 32, 1500
    b = _blocks(kind, 57, [most] * rows, 8, 128)
    space = pgcm.KVWorkspace()
    pgcm.kv_window_reserve(space, 16, 8, 128)
    tables, lens = b.r.gpu_tables()
    q = _q(58, rows, 16, 128, kind[0]).cuda()
    outs = [torch.zeros_like(q) for _ in range(3)]
    cache = b.cache(pgcm)

    def call(out, n=rows):
        b.call(pgcm)(cache, q[:n], tables[:n], lens[:n], out[:n], window=1000, sinks=4, workspace=space)

    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[0])
    for turn in range(4):
        lens.copy_(torch.tensor([[most, 0, 700, 17][(i * turn + i // 3) % 4] for i in range(rows)], dtype=torch.int32))
        call(outs[1])
        graph.replay()
        call(outs[2], 3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]), turn
        outs[0].fill_(3)


@kinds
def test_many_requests(kind):
    """more than 64, and more than are cut into parts"""
    for n, most in ((150, 900), (600, 400)):
        lens = [(37 * i) % most for i in range(n)]
        b = _blocks(kind, 11, lens, 1, 64)
        ref.check(pgcm, b, _q(12, n, 2, 64, kind[0]), [1] * n, 300, 8)


@kinds
@pytest.mark.parametrize("window, sinks", [(0, 0), (1, 0), (30, 5), (64, 64), (500, 0)])
def test_new_tokens(kind, window, sinks):
    """several of a request, of none, more than the request has, and rows that no request has"""
    lens, news = [300, 5, 0, 129, 64, 17], [7, 9, 2, 0, 64, 17]
    b = _blocks(kind, 13, lens, 2, 128)
    ref.check(pgcm, b, _q(14, sum(news), 8, 128, kind[0]), news, window, sinks, spare=5, most=64)


@pytest.mark.parametrize("half", HALVES)
@pytest.mark.parametrize("kv, group, dim, block", [(1, 1, 8, 16), (3, 5, 64, 32), (2, 16, 80, 48), (2, 17, 128, 64), (1, 40, 256, 16),
                                                   (1, 3, 144, 16), (8, 1, 120, 16), (1, 2, 48, 4096), (1, 130, 24, 16)])
def test_rows_of_all_heads_and_sizes(half, kv, group, dim, block):
    lens, news = [300, 70, 0, 500], [150, 70, 3, 90]
    b = ref.Blocks(41, lens, kv, dim, half, block=block, holes=0.1 if block == 16 else 0.0)
    q = _q(42, sum(news), kv * group, dim, half)
    for window, sinks in ((0, 0), (100, 20), (3, 0)):
        ref.check(pgcm, b, q, news, window, sinks, spare=1)


@pytest.mark.parametrize("half", HALVES)
@pytest.mark.parametrize("lens, news, kv, group, dim, window, sinks", [
    ([9000, 800], [40, 100], 2, 4, 128, 0, 0), ([9000, 800], [40, 100], 2, 4, 128, 5000, 700), ([20000], [2], 1, 1, 64, 0, 0),
    ([7001], [200], 1, 3, 256, 6000, 3), ([4000, 33, 4100], [5, 33, 8], 1, 8, 80, 0, 0), ([6000], [64], 1, 4, 128, 1500, 4)])
def test_rows_in_parts(half, lens, news, kv, group, dim, window, sinks):
    """few rows and much to see: cut along what they see, with holes"""
    b = ref.Blocks(43, lens, kv, dim, half, holes=0.2)
    ref.check(pgcm, b, _q(44, sum(news), kv * group, dim, half), news, window, sinks, spare=2)


@kinds
def test_lengths_out_of_range(kind):
    """beyond the row's blocks: cut to them; below zero: none"""
    b = _blocks(kind, 45, [47, 31, 16], 2, 64)      # rows of three blocks and one more
    for news in ([1, 1, 1], [20, 3, 2]):
        q = _q(46, sum(news), 4, 64, kind[0]).cuda()
        starts = torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32).cuda()
        tables = torch.from_numpy(b.tables).cuda()
        tables[:, 3:] = -1
        outs = []
        for lens in ([1 << 30, -7, 16], [64, 0, 16]):
            out = torch.zeros_like(q)
            b.call(pgcm)(b.cache(pgcm), q, tables, torch.tensor(lens, dtype=torch.int32).cuda(), out, window=20, sinks=3,
                         starts=starts, most=max(news))
            outs.append(out)
        assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
        assert bool((outs[0][news[0]:news[0] + news[1]] == 0).all())


@kinds
def test_on_another_stream(kind):
    b = _blocks(kind, 47, [3000, 200], 2, 128)
    stream = torch.cuda.Stream()
    for news in ([1, 1], [30, 4]):
        q = _q(48, sum(news), 8, 128, kind[0])
        want = ref.run(pgcm, b, q, news, 1000, 4)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            got = ref.run(pgcm, b, q, news, 1000, 4)
        stream.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("half", HALVES)
def test_random_shapes_of_many_rows(half):
    """requests, rows, windows, sinks and holes at random, against the definition"""
    import random
    rng = random.Random(49)
    for case in range(14):
        kv, group = rng.choice([(1, 1), (2, 4), (1, 7), (3, 2), (1, 16)])
        dim, block = rng.choice([64, 80, 128, 128, 256]), rng.choice([16, 32, 64])
        lens = [rng.choice([0, 1, rng.randint(1, 80), rng.randint(1, 700)]) for _ in range(rng.randint(1, 5))]
        news = [rng.choice([0, 1, min(t + 2, rng.randint(1, 60)), min(t, 130)]) for t in lens]
        if max(news) < 2:
            news[0] = 2
        b = ref.Blocks(100 + case, lens, kv, dim, half, block=block, holes=rng.choice([0.0, 0.0, 0.3]))
        q = _q(200 + case, sum(news), kv * group, dim, half, 1.5)
        ref.check(pgcm, b, q, news, rng.choice([0, 1, rng.randint(2, 40), rng.randint(40, 500)]), rng.choice([0, 4, 33]), spare=2)


@kinds
def test_one_row_of_some_requests(kind):
    lens, news = [300, 5, 0, 129, 64], [1, 0, 1, 1, 0]
    b = _blocks(kind, 15, lens, 2, 128)
    ref.check(pgcm, b, _q(16, 3, 8, 128, kind[0]), news, 40, 4, spare=3, most=1)


@kinds
def test_starts_beyond_the_rows(kind):
    """cut to the rows, and to the most of a request; nothing else is written"""
    b = _blocks(kind, 17, [50, 60, 70], 2, 64)
    q = _q(18, 9, 4, 64, kind[0])
    got, lse = ref.run(pgcm, b, q, [4, 3, 2], starts=[-3, 4, 7, 900], most=4)
    same, same_lse = ref.run(pgcm, b, q, [4, 3, 2], most=4)
    assert torch.equal(got, same) and torch.equal(lse, same_lse)
    got, lse = ref.run(pgcm, b, q, [4, 3, 2], starts=[0, 4, 7, 9], most=2)
    want_out, want_lse = ref.attend(b, q[[0, 1, 4, 5, 7, 8]], [2, 2, 2], 0.125, 0, 0, kind[1] is None)
    ref16.within(got[[0, 1, 4, 5, 7, 8]], want_out, "out")
    assert bool((got[[2, 3, 6]] == 7).all()) and bool((lse[[2, 3, 6]] == 7).all())


@kinds
@pytest.mark.parametrize("order", ["btkd", "bktd", "kbtd"])
def test_layouts(kind, order):
    if kind[1] is not None:
        b = _blocks(kind, 19, [200, 90], 3, 128, pieces=order == "btkd")
    else:
        b = _blocks(kind, 19, [200, 90], 3, 128, order=order)
    for news in ([1, 1], [40, 3]):
        ref.check(pgcm, b, _q(20, sum(news), 6, 128, kind[0]), news, 64, 4)


@kinds
def test_scores_of_all_sizes(kind):
    """large scores of both signs, a scale of zero"""
    b = _blocks(kind, 21, [400, 33, 1], 2, 128)
    for news in ([1, 1, 1], [50, 20, 1]):
        q = _q(22, sum(news), 4, 128, kind[0])
        for scale in (3.0, -0.5, 0.0):
            ref.check(pgcm, b, q, news, 0, 0, scale=scale)


@kinds
def test_queries_of_all_sizes(kind):
    """the largest, tiny ones, and zeros"""
    b = _blocks(kind, 23, [100] * 5, 1, 64)
    q = _q(24, 5, 2, 64, kind[0])
    top = torch.finfo(kind[0]).max
    for i, f in enumerate((2.0 ** -12, 2.0 ** -14 if kind[0] == torch.float16 else 2.0 ** -100, 0.0, 1.0, 2.0 ** 12)):
        q[i] *= f
    q[3, 0, 5] = top / 4
    ref.check(pgcm, b, q, [1] * 5, 0, 0, scale=2.0 ** -13)


@pytest.mark.parametrize("half", HALVES)
def test_values_that_are_not_finite_stay_in_rows_that_see_them(half):
    lens, news = [300, 200, 100], [200, 1, 60]
    for news in ([200, 1, 60], [1, 1, 1]):
        b = ref.Blocks(25, lens, 2, 128, half)
        q = _q(26, sum(news), 8, 128, half)
        window, sinks = 90, 5
        clean, _ = ref.run(pgcm, b, q, news, window, sinks)
        places = {0: [3, 150, 280, 299], 1: [199, 20], 2: [70, 2]}
        for i, at in places.items():
            for n, t in enumerate(at):
                block = int(b.tables[i, t // 16])
                b.r.v[block, t % 16, n % 2, 10 + n] = (math.inf, math.nan, -math.inf)[n % 3]
        got, _ = ref.run(pgcm, b, q, news, window, sinks)
        row = 0
        touched = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
        for i, c in enumerate(news):
            for j in range(c):
                end = lens[i] - (c - 1 - j)
                for n, t in enumerate(places[i]):
                    if t < end and (t >= end - window or t < sinks):
                        touched[row, 4 * (n % 2):4 * (n % 2) + 4, 10 + n] = True
                row += 1
        assert not bool(torch.isfinite(got[touched]).any())
        assert torch.equal(got[~touched], clean[~touched])


@pytest.mark.parametrize("half", HALVES)
def test_keys_that_are_not_finite(half):
    lens = [100, 100, 100, 100]
    for news in ([1] * 4, [30] * 4):
        b = ref.Blocks(27, lens, 1, 64, half)
        q = _q(28, sum(news), 2, 64, half).abs() + 0.5
        clean, clean_lse = ref.run(pgcm, b, q, news, 40, 4)
        for i, (t, x) in enumerate([(95, -math.inf), (95, math.inf), (95, math.nan), (30, math.nan)]):
            b.r.k[int(b.tables[i, t // 16]), t % 16, 0, 7] = x
        got, lse = ref.run(pgcm, b, q, news, 40, 4)
        n = news[0]
        sees = [100 - (n - 1 - j) > 95 for j in range(n)]      # the token at place 95
        for i in range(4):
            rows = slice(i * n, (i + 1) * n)
            for j in range(n):
                x = got[i * n + j]
                if i in (1, 2) and sees[j] or i == 3 and 100 - (n - 1 - j) - 40 <= 30:
                    assert bool(torch.isnan(x).all())
                elif i == 0 and sees[j]:
                    assert bool(torch.isfinite(x).all()) and not torch.equal(x, clean[i * n + j])
                else:
                    assert torch.equal(x, clean[i * n + j]), (i, j)
            del rows


def test_scales_that_are_no_numbers():
    """a block whose scale is NaN makes its head's results NaN where it is seen"""
    for code in ref8.CODES:
        b = ref.Blocks8(29, [200, 200], 2, 64, torch.bfloat16, code)
        q = _q(30, 2, 4, 64, torch.bfloat16)
        clean, _ = ref.run(pgcm, b, q, [1, 1], 50, 16)
        b.parts[2][int(b.tables[0, 11]), 1] = math.nan      # seen by the second head's queries
        b.parts[3][int(b.tables[1, 3]), 0] = math.nan       # not seen
        got, _ = ref.run(pgcm, b, q, [1, 1], 50, 16)
        assert bool(torch.isnan(got[0, 2:]).all())
        assert torch.equal(got[0, :2], clean[0, :2]) and torch.equal(got[1], clean[1])


@kinds
def test_two_calls_on_one_workspace_and_a_graph(kind):
    """a captured call, replayed with other lengths and queries between eager calls of other shapes"""
    b = _blocks(kind, 31, [5000, 900, 17], 2, 128)
    space = pgcm.KVWorkspace()
    pgcm.kv_window_reserve(space, 16, 2, 128)
    tables, lens = b.r.gpu_tables()
    news = [1, 1, 1] if kind[1] is not None else [40, 1, 5]
    rows = sum(news)
    starts = torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32).cuda()
    q = torch.zeros(rows, 8, 128, dtype=kind[0], device="cuda")
    outs = [torch.zeros_like(q) for _ in range(2)]
    cache = b.cache(pgcm)

    def call(out):
        b.call(pgcm)(cache, q, tables, lens, out, window=3000, sinks=4, starts=starts, most=max(news), workspace=space)

    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[0])
    for turn in range(4):
        q.copy_(_q(40 + turn, rows, 8, 128, kind[0]).cuda())
        lens.copy_(torch.tensor([[5000, 900, 17], [4000, 0, 60], [1, 1, 1], [4999, 33, 12]][turn], dtype=torch.int32))
        call(outs[1])
        graph.replay()
        torch.cuda.synchronize()
        # (bits, as a length of 60 takes in what is no number)
        assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)), turn
        outs[0].fill_(3)


def test_without_room_a_captured_call_is_refused():
    b = ref.Blocks(33, [5000], 2, 128, torch.float16)
    space = pgcm.KVWorkspace()
    tables, lens = b.r.gpu_tables()
    q = _q(34, 1, 4, 128, torch.float16).cuda()
    out, cache = torch.zeros_like(q), b.cache(pgcm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(pgcm.PgcmError):
        with torch.cuda.graph(graph):
            pgcm.kv_window(cache, q, tables, lens, out, workspace=space)
    torch.cuda.synchronize()
    pgcm.kv_window(cache, q, tables, lens, out, workspace=space)


def test_results_are_the_same_each_time():
    for kind in KINDS:
        b = _blocks(kind, 35, [9000, 2000, 777], 2, 128)
        for news in ([1, 1, 1], [100, 2, 30]):
            q = _q(36, sum(news), 8, 128, kind[0])
            first = ref.run(pgcm, b, q, news, 0, 0)
            for _ in range(3):
                again = ref.run(pgcm, b, q, news, 0, 0)
                assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
