"""The operators on blocks in 8 bits and attention with a window as they are used together."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2411_03357_amd as pgcm
import kv8_reference as ref8
import kv_reference as ref16
import kv_window_reference as window

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


class _State:
    """a cache as the references take it"""

    def __init__(self, k, v, tables, lens, block, kv, half):
        self.k, self.v, self.tables, self.lens, self.block, self.kv, self.half = k, v, tables, lens, block, kv, half


@pytest.mark.parametrize("code", ref8.CODES)
@pytest.mark.parametrize("half", [torch.float16, torch.bfloat16])
def test_a_prompt_and_steps_in_eight_bits(half, code):
    """a prompt in chunks is appended in 8 bits and attended to as it reads back; then steps attend over the codes.  Codes as
    their definition has them, to the last bit, and attention in 64 bits over them"""
    n, kv, heads, dim, block, row = 2, 2, 8, 64, 16, 20
    win, sinks = 70, 4
    blocks = n * row
    cpu = ref8.pool8(1, blocks, block, kv, dim, code)
    gpu = ref8.on_gpu(cpu, block, kv, dim, code, True)
    cache8 = pgcm.KV8Cache(*gpu, half)
    halves = torch.zeros(blocks, 2, block, kv, dim, dtype=half, device="cuda")
    cache = pgcm.KVCache(halves[:, 0], halves[:, 1])
    tables = np.random.default_rng(2).permutation(blocks).astype(np.int32).reshape(n, row)
    on_tables = torch.from_numpy(tables).cuda()
    want = [ref8.Blocks8(cpu[i], cpu[2 + i]) for i in (0, 1)]
    lens = np.zeros(n, np.int32)
    for step, news in enumerate([(90, 37), (50, 64), (1, 1), (1, 1), (3, 0), (1, 1)] + [(1, 1)] * 20):
        total = sum(news)
        x = ref16.numbers(100 + step, total, heads + 2 * kv, dim).to(half)
        x[:, heads:] *= 2.0 ** (step % 3)
        slots, positions = [], []
        for b in range(n):
            at = np.arange(lens[b], lens[b] + news[b])
            slots += list(tables[b, at // block].astype(np.int64) * block + at % block)
            row0 = sum(news[:b])
            for i in (0, 1):
                y = x[row0:row0 + news[b], heads + i * kv:heads + (i + 1) * kv].double().numpy()
                for j in sorted(set(at // block)):
                    mine = at // block == j
                    want[i].append(tables[b, j], int(at[mine][0] % block), y[mine])
            lens[b] += news[b]
        on = x.cuda()
        pgcm.kv8_append(cache8, None, on[:, heads:heads + kv], on[:, heads + kv:], None, torch.tensor(slots).cuda(), None)
        for i in (0, 1):
            want[i].same(gpu[i], gpu[2 + i], "step %d" % step)
        q, out = on[:, :heads], torch.zeros(total, heads, dim, dtype=half, device="cuda")
        on_lens = torch.from_numpy(lens).cuda()
        starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()
        many = max(news) > 1
        if many:
            used = torch.from_numpy(np.concatenate([tables[b, :-(-int(lens[b]) // block)] for b in range(n)])).cuda()
            pgcm.kv8_load(cache8, cache, used)
            pgcm.kv_window(cache, q, on_tables, on_lens, out, window=win, sinks=sinks, starts=starts, most=max(news))
        else:
            pgcm.kv8_attend(cache8, q, on_tables, on_lens, out, window=win, sinks=sinks)
        k, v = [torch.from_numpy(w.codes * w.scales[:, None, :, None]) for w in want]
        if many:    # as they read back
            k, v = [ref8.halves(y.numpy(), half).double() for y in (k, v)]
        state = _State(k, v, tables, lens.tolist(), block, kv, half)
        rounded = many
        got = window.attend(state, x[:, :heads], list(news), dim ** -0.5, win, sinks, rounded)[0]
        # (weights over codes are two halves of binary16, whatever the cache's: below 2^-37 of the largest)
        tol = got[1] + (0 if many else 2.0 ** -36 * float(v.abs().max()))
        ref16.within(out, (got[0], tol), "step %d" % step)


@pytest.mark.parametrize("code", ref8.CODES)
def test_blocks_leave_in_eight_bits_and_come_back(code):
    """examples/kv_decode.py with a code: what comes back is what left, rounded to 8 bits"""
    import kv_decode
    torch.manual_seed(4)
    d = kv_decode.Decoder(3, 3, 160, keep=3, code=code)
    left, back = {}, []
    encrypt, decrypt = d._encrypt, d._decrypt

    def watched_encrypt(places, blocks):
        left.update({p: d.pool[b].cpu() for p, b in zip(places, blocks)})
        encrypt(places, blocks)

    def watched_decrypt(places, blocks):
        decrypt(places, blocks)
        for p, b in zip(places, blocks):
            back.append((left[p], d.pool[b].cpu()))

    d._encrypt, d._decrypt = watched_encrypt, watched_decrypt
    d.prompt(*[torch.randn(3, 40, h, d.dim, device="cuda").to(d.half) for h in (8, 2, 2)])
    for step in range(110):
        d.step(*[torch.randn(3, h, d.dim, device="cuda").to(d.half) for h in (8, 2, 2)])
        if step % 30 == 29:
            d.recall()
    assert d.chunk == 2 * 16 * 2 * 128 + 16 and d.moved["out"] > 9 and len(back) > 3
    cpu = ref8.pool8(1, 1, 16, 2, 128, code)
    for before, after in back:
        for i in (0, 1):
            want = ref8.Blocks8(cpu[i], cpu[2 + i])
            want.start(0, before[i].double().numpy())
            assert torch.equal(after[i], ref8.halves(want.codes[0] * want.scales[0][:, None], d.half))


def test_the_example_runs_with_prompts_and_eight_bits():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "kv_decode.py"), "--steps", "60", "--prompt", "100",
                          "--leave", "int8"], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=100)
    assert out.returncode == 0, out.stderr[-1500:]
    assert "all authentic" in out.stdout


def test_a_prompt_attends_as_its_definition_says():
    import kv_decode
    torch.manual_seed(5)
    d = kv_decode.Decoder(2, 30, 200, window=30, sinks=3)
    for new in (50, 1, 33):
        q, k, v = [torch.randn(2, new, h, d.dim, device="cuda").to(d.half) for h in (8, 2, 2)]
        out = d.prompt(q, k, v)
        state = _State(d.pool[:, 0].cpu().double(), d.pool[:, 1].cpu().double(), d.tables, d.lens.tolist(), d.block, 2, d.half)
        want = window.attend(state, d.q.cpu(), [new, new], d.dim ** -0.5, 30, 3, new > 1)[0]
        ref16.within(out.flatten(0, 1), want, "prompt of %d" % new)


def test_a_captured_step():
    """an append in 8 bits, its attention, the read-back and attention over halves in one graph, replayed with other values"""
    half, code = torch.bfloat16, torch.float8_e4m3fn
    n, kv, heads, dim, block, row = 3, 2, 8, 128, 16, 200
    cpu = ref8.pool8(3, n * row, block, kv, dim, code)
    sides = []
    for _ in range(2):
        gpu = ref8.on_gpu(cpu, block, kv, dim, code, True)
        pool = torch.zeros(n * row, 2, block, kv, dim, dtype=half, device="cuda")
        sides.append((gpu, pgcm.KV8Cache(*gpu, half), pool, pgcm.KVCache(pool[:, 0], pool[:, 1]),
                      [torch.zeros(n, heads, dim, dtype=half, device="cuda") for _ in range(3)]))
    tables = torch.arange(n * row, dtype=torch.int32, device="cuda").view(n, row)
    every = tables.flatten().contiguous()
    lens, slots = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda")
    positions = torch.zeros_like(lens)
    packed = torch.zeros(n, heads + 2 * kv, dim, dtype=half, device="cuda")
    rope = torch.randn(4096, dim, device="cuda")
    space = pgcm.KVWorkspace()
    pgcm.kv_window_reserve(space, heads, kv, dim)

    def step(side):
        _, cache8, _, cache, (q, out, out16) = side
        pgcm.kv8_append(cache8, packed[:, :heads], packed[:, heads:heads + kv], packed[:, heads + kv:], positions, slots, q, rope=rope)
        pgcm.kv8_attend(cache8, q, tables, lens, out, window=1000, sinks=2, workspace=space)
        pgcm.kv8_load(cache8, cache, every)
        pgcm.kv_window(cache, q, tables, lens, out16, workspace=space)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sides[0])
    for turn, now in enumerate(([3000, 5, 3200], [3001, 1, 17], [64, 3199, 2000])):
        packed.copy_(ref16.numbers(50 + turn, *packed.shape).to(half))
        at = torch.tensor(now).cuda() - 1
        lens.copy_(at + 1)
        positions.copy_(at)
        slots.copy_(tables.gather(1, (at // block)[:, None])[:, 0] * block + at % block)
        step(sides[1])
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(sides[0][4], sides[1][4]):
            assert torch.equal(x, y)
        assert torch.equal(sides[0][2], sides[1][2])
        for x, y in zip(sides[0][0], sides[1][0]):
            assert torch.equal(x.float(), y.float())
    space.destroy()


def test_offsets_beyond_32_bits():
    """blocks that lie gigabytes apart: all operators against the same on blocks close together"""
    half, code, block, kv, dim, heads = torch.float16, torch.int8, 16, 2, 64, 4
    apart8, apart16 = 3 << 30, 3 << 30      # codes; halves
    whole = torch.empty(2 * apart8 + (1 << 20), dtype=torch.uint8, device="cuda")
    whole16 = torch.empty(2 * apart16 + (1 << 20), dtype=half, device="cuda")
    inner = (kv * dim, dim, 1)
    size = block * kv * dim
    far = [whole.view(code).as_strided((3, block, kv, dim), (apart8, *inner), i * size) for i in (0, 1)]
    far += [whole.view(torch.float32).as_strided((3, kv), (apart8 // 4, 1), (2 * size + 16 * i) // 4) for i in (0, 1)]
    far16 = [whole16.as_strided((3, block, kv, dim), (apart16, *inner), i * size) for i in (0, 1)]
    near = ref8.on_gpu(ref8.pool8(5, 3, block, kv, dim, code), block, kv, dim, code, True)
    near16 = torch.zeros(3, 2, block, kv, dim, dtype=half, device="cuda")
    x = ref16.numbers(6, 40, heads + 2 * kv, dim).to(half).cuda()
    tables, lens = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda(), torch.tensor([40], dtype=torch.int32).cuda()
    slots = torch.tensor([32 + t if t < 16 else t - 16 if t < 32 else t - 16 for t in range(40)]).cuda()
    starts = torch.tensor([0, 40], dtype=torch.int32).cuda()
    every = torch.arange(3, dtype=torch.int32, device="cuda")
    got = []
    for parts, halves in ((far, far16), (near, [near16[:, 0], near16[:, 1]])):
        cache8, cache = pgcm.KV8Cache(*parts, half), pgcm.KVCache(*halves)
        outs = [torch.zeros(1, heads, dim, dtype=half, device="cuda"), torch.zeros(1, heads, dim, dtype=half, device="cuda"),
                torch.zeros(40, heads, dim, dtype=half, device="cuda")]
        pgcm.kv8_append(cache8, None, x[:, heads:heads + kv], x[:, heads + kv:], None, slots, None)
        pgcm.kv8_attend(cache8, x[39:, :heads], tables, lens, outs[0])
        pgcm.kv8_load(cache8, cache, every)
        pgcm.kv_window(cache, x[39:, :heads], tables, lens, outs[1])
        pgcm.kv_window(cache, x[:, :heads], tables, lens, outs[2], starts=starts, most=40)
        halves[0][:, 3] *= 3
        pgcm.kv8_store(cache8, cache, every, torch.tensor([16, 8, 16], dtype=torch.int32).cuda())
        got.append(outs + [p.float().clone() for p in parts])
    for a, b in zip(*got):
        rows = slice(None) if a.dim() != 4 else [0, 2]      # (the third block's last places are anything)
        assert torch.equal(a[rows], b[rows])
