"""Attention with a window from its definition, on the CPU, in 64 bits.  Shares nothing with the library."""
import math

import numpy as np
import torch

import kv8_reference as ref8
import kv_reference as ref16


class Blocks:
    """Requests on blocks of halves: what they may read as numbers in 64 bits, and the cache on the device."""

    def __init__(self, seed, lens, kv, dim, half, block=16, holes=0.0, order="btkd", junk=math.nan):
        self.r = ref16.Requests(seed, lens, kv, dim, half, block, holes, junk, order)
        self.k, self.v = self.r.k.double(), self.r.v.double()
        self.tables, self.lens, self.block, self.kv, self.half = self.r.tables, self.r.lens, block, kv, half

    def cache(self, pgcm):
        return pgcm.KVCache(*self.r.on_gpu())

    def call(self, pgcm):
        return pgcm.kv_window


class Blocks8(Blocks):
    """... on blocks in 8 bits.  Places and scales that no request may read hold what is no number, where there is such a thing."""

    def __init__(self, seed, lens, kv, dim, half, code, block=16, holes=0.0, pieces=True):
        super().__init__(seed, lens, kv, dim, half, block, holes)
        owned = torch.zeros(self.r.blocks, dtype=torch.bool)
        owned[torch.from_numpy(self.tables[self.tables >= 0]).long()] = True
        self.parts = list(ref8.pool8(seed, self.r.blocks, block, kv, dim, code, pieces))
        junk = 0x7F if code == torch.float8_e4m3fn else 0x80
        for i, x in enumerate((self.k, self.v)):
            there = ~torch.isnan(x)
            bits = self.parts[i].view(torch.uint8)
            bits.copy_(torch.where(there, bits, torch.tensor(junk, dtype=torch.uint8)))
            # about as large as normal numbers: e4m3's are larger than int8's on the whole
            self.parts[2 + i].copy_(2.0 ** torch.from_numpy(np.random.default_rng([82, seed, i]).integers(-8, -4, (self.r.blocks, kv))) *
                                    (1.25 if i else 0.75))
            self.parts[2 + i][~owned] = math.nan
            values = self.parts[i].double() if code == torch.int8 else self.parts[i].float().double()
            x.copy_(torch.where(there, values * self.parts[2 + i].double()[:, None, :, None], x))
        self.code, self.dim, self.pieces = code, dim, pieces

    def cache(self, pgcm):
        return pgcm.KV8Cache(*ref8.on_gpu(self.parts, self.block, self.kv, self.dim, self.code, self.pieces), self.half)

    def call(self, pgcm):
        return pgcm.kv8_attend


def attend(b, q, news, scale, window, sinks, rounded):
    """out and lse of q's rows in 64 bits, and for each how far it may be off.

    A score is off by at most e = (dim + 6) 2^-24 scale sum |q k|; a weight by 2 e, and by what n additions (n 2^-24), the
    exponential and its argument (2^-22 of the largest) make of it; `rounded`: and by a rounding to a half, in binary16 by
    2^-25 of the largest weight at least.  Not rounded: by 2^-22, and where weights are two halves of binary16, of which the
    largest's first is at least 2^13 and the least that a half can tell apart 2^-24, by half of that, 2^-38 of the largest (which
    counts where the values of large weights are zero)."""
    q = q.double()
    rows, heads, dim = q.shape
    group = heads // b.kv
    out, lse = torch.full((rows, heads, dim), 7.0, dtype=torch.float64), torch.full((rows, heads), 7.0, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    row = 0
    for i, n_new in enumerate(news):
        length = max(0, min(b.lens[i], b.tables.shape[1] * b.block))
        for j in range(n_new):
            end = length - (n_new - 1 - j)
            out[row], lse[row] = 0.0, -math.inf
            seen = [t for t in range(max(0, end)) if (window == 0 or t >= end - window or t < sinks) and
                    0 <= b.tables[i, t // b.block] < b.k.shape[0]]
            if seen:
                t = torch.tensor(seen)
                at = torch.from_numpy(b.tables[i])[t // b.block].long()
                for g in range(b.kv):
                    k, v = b.k[at, t % b.block, g], b.v[at, t % b.block, g]
                    mine = slice(g * group, (g + 1) * group)
                    s = (q[row, mine] @ k.T) * scale
                    e = ((dim + 6) * 2.0 ** -24 * abs(scale) * (q[row, mine].abs() @ k.abs().T)).amax(1)
                    lse[row, mine] = torch.logsumexp(s, 1)
                    p = (s - lse[row, mine, None]).exp()
                    off = 2 * e + (len(seen) + 16) * 2.0 ** -24 + 2.0 ** -22 * (s.abs().amax(1) * 1.5 + 4)
                    size = p @ v.abs()
                    more = 2.0 ** -21 * size
                    if isinstance(b, Blocks8) or b.half == torch.float16:
                        more = more + 2.0 ** -38 * p.amax(1, keepdim=True) * v.abs().sum(0)
                    if rounded:
                        more = ref16.UNIT[b.half] * size + ref16.LEAST[b.half] * p.amax(1, keepdim=True) * v.abs().sum(0)
                    lse_tol[row, mine] = off
                    out[row, mine] = p @ v
                    out_tol[row, mine] = ref16.UNIT[b.half] * out[row, mine].abs() + ref16.LEAST[b.half] + \
                        (off[:, None] * size + more) * 1.01
            row += 1
    return (out, out_tol), (lse, lse_tol)


def run(pgcm, b, q, news, window=0, sinks=0, starts=None, most=None, scale=None, spare=0, **more):
    """out and lse of a call; rows behind the last request's, `spare` of them, hold 7 before it"""
    rows, heads, dim = q.shape
    on = torch.full((rows + spare, heads + 1, dim), math.nan, dtype=b.half, device="cuda")[:, :heads]
    on[:rows] = q.cuda()
    out = torch.full((rows + spare, heads, dim), 7.0, dtype=b.half, device="cuda")
    lse = torch.full((rows + spare, heads), 7.0, device="cuda")
    if starts is None and news != [1] * len(news):
        starts = np.concatenate([[0], np.cumsum(news)])
    if starts is not None:
        starts = torch.tensor(np.asarray(starts), dtype=torch.int32).cuda()
    tables, lens = b.r.gpu_tables()
    b.call(pgcm)(b.cache(pgcm), on, tables, lens, out, lse=lse, scale=scale, window=window, sinks=sinks, starts=starts, most=most,
                 **more)
    return out, lse


def check(pgcm, b, q, news, window=0, sinks=0, scale=None, rounded=None, **more):
    out, lse = run(pgcm, b, q, news, window, sinks, scale=scale, **more)
    rows = q.shape[0]
    if rounded is None:
        rounded = not isinstance(b, Blocks8) and max(news) > 1
    want_out, want_lse = attend(b, q, news, q.shape[2] ** -0.5 if scale is None else scale, window, sinks, rounded)
    what = "window %d sinks %d" % (window, sinks)
    ref16.within(out[:rows], want_out, "out, " + what)
    ref16.within(lse[:rows], want_lse, "lse, " + what)
    assert bool((out[rows:] == 7).all()) and bool((lse[rows:] == 7).all())
    return out, lse
