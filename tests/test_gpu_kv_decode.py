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
