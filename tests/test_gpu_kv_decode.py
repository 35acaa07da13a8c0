"""The operators and the cipher on the same blocks (examples/kv_decode.py), step by step against a cache that never leaves."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


class _Shadow:
    """every key and value that was ever appended, in blocks of its own: block request * row + place"""

    def __init__(self, d):
        self.d, self.half, self.block, self.kv, self.dim, self.most = d, d.half, d.block, d.kv_heads, d.dim, d.row
        self.blocks = d.n * d.row
        self.k = torch.zeros(self.blocks, d.block, d.kv_heads, d.dim, dtype=d.half)
        self.v = torch.zeros_like(self.k)

    def append(self):
        """takes the newest token as the cache has it"""
        for b in range(self.d.n):
            t = int(self.d.lens[b]) - 1
            j = t // self.block
            row = self.d.pool[int(self.d.tables[b, j]), :, t % self.block].cpu()
            self.k[b * self.most + j, t % self.block], self.v[b * self.most + j, t % self.block] = row[0], row[1]

    def where(self, present):
        at = np.arange(self.blocks, dtype=np.int32).reshape(self.d.n, self.most)
        self.tables, self.lens = np.where(present, at, -1), self.d.lens.tolist()
        return self


def test_decoding_with_blocks_that_come_and_go():
    import kv_decode
    torch.manual_seed(3)
    d = kv_decode.Decoder(3, 3, 160, keep=3)
    shadow = _Shadow(d)
    weights = torch.zeros(3, d.row, dtype=torch.float64)
    tol = torch.zeros_like(weights)
    for step in range(150):
        q, k, v = [torch.randn(3, h, d.dim, device="cuda").to(d.half) for h in (8, 2, 2)]
        before = d.tables.copy()
        out = d.step(q, k, v)
        present = before >= 0
        present[np.arange(3), (d.lens - 1) // d.block] = True     # attended over before any of them left
        if d.tables[0, (d.lens[0] - 1) // d.block] >= 0:
            shadow.append()
        want = ref.attend(shadow.where(present), d.q.cpu(), d.dim ** -0.5)
        if step % 10 == 9:
            ref.within(out, want[0], "out of step %d" % step)
        weights, tol = 0.98 * weights + want[2][0], 0.98 * tol + want[2][1] + 2.0 ** -22 * weights
        if step % 50 == 49:
            out, selected = d.recall()
            got = ref.attend(shadow.where(np.ones_like(present)), d.q.cpu(), d.dim ** -0.5, selected)
            ref.within(out, got[0], "recalled at step %d" % step)
            kept = {(b, j): int(d.tables[b, j]) for b in range(3) for j in range(d.row) if d.tables[b, j] >= 0}
            for (b, j), block in kept.items():      # what came back is what left, to the last bit
                n = min(d.block, int(d.lens[b]) - j * d.block)
                assert torch.equal(d.pool[block, 0, :n].cpu(), shadow.k[b * d.row + j, :n])
                assert torch.equal(d.pool[block, 1, :n].cpu(), shadow.v[b * d.row + j, :n])
    ref.within(d.weights, (weights, tol), "weights")
    assert d.moved["out"] > 9 and d.moved["in"] > 3
    used = [int(i) for i in d.tables.ravel() if i >= 0]
    assert len(set(used)) == len(used) and sorted(used + d.free) == list(range(d.pool.shape[0]))


def test_the_example_runs():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "kv_decode.py"), "--steps", "120"],
                         stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=100)
    assert out.returncode == 0, out.stderr[-1500:]
    assert "all authentic" in out.stdout


def test_a_step_captured_into_a_graph():
    """all operators of a decode step in one graph, replayed with other inputs, lengths and tables, against the same calls
    outside of it"""
    import paper_2411_03357_amd as pgcm
    gen = torch.Generator(device="cuda").manual_seed(5)
    n, kv, heads, dim, block, row = 2, 2, 8, 64, 16, 1300
    half = torch.bfloat16
    pool = torch.randn(n * row, 2, block, kv, dim, device="cuda", generator=gen).to(half)
    cache = pgcm.KVCache(pool[:, 0], pool[:, 1])
    tables = torch.arange(n * row, dtype=torch.int32, device="cuda").view(n, row)
    blocks = tables.flatten().contiguous()
    bounds = torch.zeros(n * row, kv, 2, dim, dtype=torch.int8, device="cuda")
    scales = torch.zeros(n * row, kv, device="cuda")
    pgcm.kv_summarize(cache, blocks, torch.full_like(blocks, block), bounds, scales)
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    positions, last, counts = torch.zeros_like(lens), torch.zeros_like(lens), torch.zeros_like(lens)
    packed = torch.zeros(n, heads + 2 * kv, dim, dtype=half, device="cuda")
    rope = torch.randn(32768, dim, device="cuda", generator=gen)
    weights = torch.zeros(n, row, device="cuda")
    q = torch.zeros(n, heads, dim, dtype=half, device="cuda")
    out, sparse = torch.zeros_like(q), torch.zeros_like(q)
    selected = torch.zeros(n, kv, 20, dtype=torch.int32, device="cuda")
    evict = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    victims = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
    space = pgcm.KVWorkspace()
    space.reserve(n, heads, kv, dim, block, row)

    def step():
        pgcm.kv_append(cache, packed[:, :heads], packed[:, heads:heads + kv], packed[:, heads + kv:], positions, slots, q,
                       rope=rope)
        pgcm.kv_summarize(cache, last, counts, bounds, scales)
        pgcm.kv_select(q, tables, lens, bounds, scales, block, selected, first=1, last=2, workspace=space)
        pgcm.kv_attend(cache, q, tables, lens, sparse, selected=selected, workspace=space)
        pgcm.kv_attend(cache, q, tables, lens, out, weights=weights, kept=weights, decay=0.9, workspace=space)
        pgcm.kv_evict(weights, tables, lens, block, evict, victims, tables_out=tables, first=1, last=2, blocks=n * row)

    changed = (pool, bounds, scales, tables, weights, q, out, sparse, selected, victims)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for now in ([20000, 700], [1, 20800], [20001, 16], [12345, 19999]):
            packed.copy_(torch.randn(packed.shape, device="cuda", generator=gen))
            at = torch.tensor(now, device="cuda") - 1
            lens.copy_(at + 1)
            positions.copy_(at)
            place = at // block
            here = tables.gather(1, place[:, None])[:, 0].long()
            slots.copy_(torch.where(here >= 0, here * block + at % block, -1))
            last.copy_(here)
            counts.copy_(at % block + 1)
            before = [x.clone() for x in changed]
            graph.replay()
            got = [x.clone() for x in changed]
            for x, y in zip(changed, before):
                x.copy_(y)
            step()
            torch.cuda.synchronize()
            for x, y in zip(changed, got):
                assert torch.equal(x, y)
            assert int((victims >= 0).sum()) > 0
    space.destroy()
