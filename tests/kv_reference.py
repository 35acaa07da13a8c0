"""The operators on KV blocks from their definitions, on the CPU: numbers in 64 bits, whole numbers exactly; and caches to
run them on.  Shares nothing with the library."""
import math

import numpy as np
import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a unit in the last place, relative
LEAST = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}           # ... below the normal numbers


def numbers(seed, *shape, std=1.0):
    return torch.from_numpy(np.random.default_rng([77, seed]).standard_normal(shape) * std)


class Requests:
    """A cache and requests on it: every place of the pool that no request may read holds `junk`.  Blocks of a request are
    absent where rng < holes.  order: strides of the pool, as the order of its dimensions in memory."""

    def __init__(self, seed, lens, kv, dim, half=torch.bfloat16, block=16, holes=0.0, junk=math.nan, order="btkd", spare=3):
        rng = np.random.default_rng([78, seed])
        self.half, self.block, self.kv, self.dim = half, block, kv, dim
        self.lens = list(lens)
        n = len(self.lens)
        self.most = max([1] + [-(-t // block) for t in self.lens]) + 1
        self.tables = np.full((n, self.most), -1, np.int32)
        there = [(b, j) for b, t in enumerate(self.lens) for j in range(-(-t // block)) if rng.random() >= holes]
        self.blocks = len(there) + spare
        ids = rng.permutation(self.blocks)
        k = np.full((self.blocks, block, kv, dim), junk)
        v = np.full((self.blocks, block, kv, dim), junk)
        for (b, j), at in zip(there, ids):
            self.tables[b, j] = at
            m = min(block, self.lens[b] - j * block)
            k[at, :m] = rng.standard_normal((m, kv, dim))
            v[at, :m] = rng.standard_normal((m, kv, dim))
        self.k, self.v = torch.from_numpy(k).to(half), torch.from_numpy(v).to(half)
        self.order = order

    def on_gpu(self):
        """k, v [block][token][head][channel] on the device, in this order in memory"""
        at = ["btkd".index(c) for c in self.order]
        back = [at.index(i) for i in range(4)]
        return [x.permute(at).contiguous().cuda().permute(back) for x in (self.k, self.v)]

    def gpu_tables(self):
        return torch.from_numpy(self.tables).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda()


def attend(r, q, scale, selected=None, kept=None, decay=1.0):
    """out, lse, weights in 64 bits, and for each how far 32-bit sums may be off: out with its rounding to half.

    A score is off by at most e = (dim + 2) 2^-24 scale sum |q k|; a weight by 2 e, and by what n additions (n 2^-24), the
    exponential and its argument (2^-22 of the largest) and two halves of 8 bits (2^-16) make of it."""
    q = q.double()
    n, heads, dim = q.shape
    group = heads // r.kv
    out, lse = torch.zeros(n, heads, dim, dtype=torch.float64), torch.full((n, heads), -math.inf, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    weights, weights_tol = torch.zeros(n, r.most, dtype=torch.float64), torch.zeros(n, r.most, dtype=torch.float64)
    for b in range(n):
        for g in range(r.kv):
            places = range(r.most) if selected is None else [int(j) for j in selected[b][g]]
            rows = [(j, t) for j in places if 0 <= j < r.most and 0 <= r.tables[b, j] < r.blocks
                    for t in range(r.block) if j * r.block + t < r.lens[b]]
            if not rows:
                continue
            at = [(int(r.tables[b, j]), t) for j, t in rows]
            k = torch.stack([r.k[i, t, g] for i, t in at]).double()
            v = torch.stack([r.v[i, t, g] for i, t in at]).double()
            mine = slice(g * group, (g + 1) * group)
            s = (q[b, mine] @ k.T) * scale
            e = ((dim + 2) * 2.0 ** -24 * abs(scale) * (q[b, mine].abs() @ k.abs().T)).amax(1)
            lse[b, mine] = torch.logsumexp(s, 1)
            p = (s - lse[b, mine, None]).exp()
            out[b, mine] = p @ v
            size = 2.0 ** -22 * (s.abs().amax(1) * 1.5 + 4)
            off = 2 * e + (len(rows) + 16) * 2.0 ** -24 + size
            lse_tol[b, mine] = off
            out_tol[b, mine] = UNIT[r.half] * out[b, mine].abs() + LEAST[r.half] + \
                (off + 2.0 ** -16)[:, None] * 1.01 * (p @ v.abs())
            for i, (j, _) in enumerate(rows):
                weights[b, j] += p[:, i].sum()
                weights_tol[b, j] += ((off + heads * 2.0 ** -24) * p[:, i]).sum()
    if kept is not None:
        weights = weights + decay * kept.double()
        weights_tol = weights_tol + 2.0 ** -22 * weights.abs()
    return (out, out_tol), (lse, lse_tol), (weights, weights_tol)


def within(got, want, what):
    value, tol = want
    got = got.double().cpu()
    assert got.shape == value.shape
    same = (got == value) | ((got - value).abs() <= tol)
    assert bool(same.all()), "%s: off by %g where %g is allowed" % (
        what, float((got - value).abs()[~same][0]), float(tol.expand_as(value)[~same][0]))


def turned(x, weight, eps, table, positions, adjacent):
    """append's norm and rotation of [tokens][heads][channels], in 64 bits"""
    x = x.double().clone()
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    if table is None:
        return x
    half = table.shape[1] // 2
    for t, at in enumerate(positions):
        row = table[at].double() if 0 <= at < table.shape[0] else torch.full((2 * half,), math.nan, dtype=torch.float64)
        c, s = row[:half], row[half:]
        first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if adjacent else (slice(0, half), slice(half, 2 * half))
        u, v = x[t, :, first].clone(), x[t, :, second].clone()
        x[t, :, first], x[t, :, second] = u * c - v * s, v * c + u * s
    return x


def eighths(rows):
    """rows of float32 in 8 bits and their scales, with the definition's roundings: numpy's float32"""
    x = np.where(np.isfinite(rows), rows, 0).astype(np.float32)
    a = np.abs(x).max(-1, keepdims=True)
    small = a < np.float32(1e-30)
    by = np.float32(127) / np.where(small, np.float32(127), a)
    whole = np.where(small, 0, np.rint(x * by)).astype(np.int64)
    return whole, np.where(small, 0, a / np.float32(127)).astype(np.float32)[..., 0]


def summarize(k, counts):
    """bounds [n][kv][2][dim] and scales [n][kv] of keys [n][tokens][kv][dim]"""
    k = k.float().numpy()
    n, block, kv, dim = k.shape
    bounds, scales = np.zeros((n, kv, 2, dim), np.int64), np.zeros((n, kv), np.float32)
    for i, m in enumerate(counts):
        m = min(max(int(m), 0), block)
        if m:
            x = np.where(np.isfinite(k[i, :m]), k[i, :m], 0)
            ends = np.stack([x.min(0), x.max(0)], 1)
            whole, scale = eighths(ends.reshape(kv, 2 * dim))
            bounds[i], scales[i] = whole.reshape(kv, 2, dim), scale
    return bounds, scales


def largest(keys, want):
    """indices of the `want` largest of (class, value) pairs, equal ones from the front, ascending"""
    return sorted(sorted(range(len(keys)), key=lambda i: (-keys[i][0], -keys[i][1], i))[:want])


def select(q, tables, lens, bounds, scales, block, keep, first, last):
    n, heads, dim = q.shape
    entries, kv = scales.shape
    group = heads // kv
    whole, qs = eighths(q.float().numpy())
    got = np.full((n, kv, keep), -1, np.int64)
    for b in range(n):
        blocks = min(-(-max(int(lens[b]), 0) // block), tables.shape[1])
        able = [j for j in range(blocks) if 0 <= tables[b, j] < entries]
        for g in range(kv):
            keys = []
            for j in able:
                c, e = whole[b, g * group:(g + 1) * group], int(tables[b, j])
                total = np.maximum(c * bounds[e, g, 0], c * bounds[e, g, 1]).sum(-1).astype(np.float32)
                score = float((total * scales[e, g] * qs[b, g * group:(g + 1) * group]).max())
                keys.append((1 if j < first or blocks - j <= last else 0, score))
            keys = [(c, 0.0 if c else s) for c, s in keys]
            at = [able[i] for i in largest(keys, keep)]
            got[b, g, :len(at)] = at
    return got


def evict(weights, tables, lens, block, asked, most, first, last, blocks):
    n, row = tables.shape
    victims = np.full((n, most), -1, np.int64)
    for b in range(n):
        have = min(-(-max(int(lens[b]), 0) // block), row)
        able = [j for j in range(first, max(0, have - last)) if 0 <= tables[b, j] < blocks]
        able = [j for j in able if j < have]
        keys = [(0, math.inf) if math.isnan(weights[b, j]) else (1, -float(weights[b, j])) for j in able]
        at = [able[i] for i in largest(keys, min(max(int(asked[b]), 0), most))]
        victims[b, :len(at)] = at
    return victims
