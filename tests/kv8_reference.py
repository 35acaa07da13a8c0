"""KV blocks in 8 bits from their definitions, on the CPU, in 64 bits.  Shares nothing with the library."""
import math

import numpy as np
import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
CODES = (torch.int8, torch.float8_e4m3fn)


def power(a, code):
    """e of the scale for a largest |x| of a"""
    e = -100
    while a > TOP[code] * 2.0 ** e:
        e += 1
    return e


def rounded(y, code):
    """the codes' values nearest to y, ties to even: whole numbers, or 4 significant bits down to steps of 2^-9"""
    if code == torch.int8:
        return np.rint(y)
    with np.errstate(divide="ignore"):
        ex = np.floor(np.log2(np.abs(np.where(y == 0, 1.0, y))))
    ex = np.where(np.abs(y) >= 2.0 ** (ex + 1), ex + 1, np.where(np.abs(y) < 2.0 ** ex, ex - 1, ex))
    step = 2.0 ** (np.maximum(ex, -6) - 3)
    return np.rint(y / step) * step


class Blocks8:
    """One kind's codes' values [block][token][head][channel] and scales [block][head] of a cache in 8 bits; start() and append()
    are what store and append make of them."""

    def __init__(self, codes, scales):
        self.code = codes.dtype
        self.codes = codes.float().numpy().astype(np.float64)
        self.scales = scales.numpy().astype(np.float64)

    def start(self, block, x):
        self._write(block, 0, x, np.zeros(x.shape[1]))

    def append(self, block, inside, x):
        """x [tokens][head][channel] from place `inside` on"""
        self._write(block, inside, x, self.scales[block].copy() if inside else np.zeros(x.shape[1]))

    def _write(self, block, inside, x, before):
        for h in range(x.shape[1]):
            a = np.abs(x[:, h]).max() if x.shape[0] else 0.0
            new = math.nan if not math.isfinite(a) or math.isnan(before[h]) else max(2.0 ** power(a, self.code), before[h])
            if inside and new == new and new != before[h]:
                self.codes[block, :inside, h] = rounded(self.codes[block, :inside, h] * (before[h] / new), self.code)
            self.codes[block, inside:inside + x.shape[0], h] = 0.0 if new != new else rounded(x[:, h] / new, self.code)
            self.scales[block, h] = new

    def same(self, codes, scales, what=""):
        got, s = codes.float().cpu().numpy(), scales.cpu().numpy()
        np.testing.assert_array_equal(s, self.scales.astype(np.float32), err_msg=what + " scales")
        np.testing.assert_array_equal(got, self.codes.astype(np.float32), err_msg=what + " codes")


def pool8(seed, blocks, block, kv, dim, code, pieces=True, heads_first=False):
    """(k, v, k_scales, v_scales) on the CPU: any codes, scales around 2^-5.  pieces: a block's codes and scales are in one
    piece, as the cipher takes them; else each is a tensor of its own."""
    rng = np.random.default_rng([81, seed])
    n = block * kv * dim
    if not pieces:
        got = [torch.empty(blocks, kv, block, dim, dtype=torch.uint8).transpose(1, 2) if heads_first else
               torch.empty(blocks, block, kv, dim, dtype=torch.uint8) for _ in "kv"]
        got = [g.view(code) for g in got]
        scales = [torch.empty(blocks, kv) for _ in "kv"]
    else:
        size = 2 * n + -(-8 * kv // 16) * 16
        whole = torch.empty(blocks, size, dtype=torch.uint8)
        got, scales = views(whole, block, kv, dim, code)
    for g in got:
        bits = rng.integers(0, 256, (blocks, block, kv, dim)).astype(np.uint8)
        bits[(bits & 0x7F) == 0x7F] = 3     # (NaN in e4m3)
        bits[bits == 0x80] = 5
        g.view(torch.uint8).copy_(torch.from_numpy(bits))
    for s in scales:
        s.copy_(torch.from_numpy(2.0 ** rng.integers(-8, -2, (blocks, kv))))
    return got[0], got[1], scales[0], scales[1]


def views(whole, block, kv, dim, code):
    """codes and scales of blocks in one piece [blocks][bytes]"""
    n = block * kv * dim
    codes = [whole[:, i * n:(i + 1) * n].view(code).unflatten(1, (block, kv, dim)) for i in (0, 1)]
    scales = [whole[:, 2 * n + 4 * i * kv:2 * n + 4 * (i + 1) * kv].view(torch.float32) for i in (0, 1)]
    return codes, scales


def on_gpu(parts, block, kv, dim, code, pieces):
    """the same on the device, laid out the same"""
    if not pieces:
        return [p.cuda() if p.is_contiguous() else p.transpose(1, 2).contiguous().cuda().transpose(1, 2) for p in parts]
    k = parts[0]
    whole = torch.empty(k.shape[0], 2 * block * kv * dim + -(-8 * kv // 16) * 16, dtype=torch.uint8, device="cuda")
    codes, scales = views(whole, block, kv, dim, code)
    for to, of in zip(codes + scales, parts):
        to.view(torch.uint8).copy_(of.view(torch.uint8))
    return codes + scales


def halves(values, half):
    """64-bit values as halves, those of finite values beyond the range as the largest"""
    top = torch.finfo(half).max
    x = torch.from_numpy(values)
    got = x.to(half) if half == torch.bfloat16 else x.float().to(half)
    return torch.where(torch.isinf(got.float()) & torch.isfinite(x), torch.sign(x).to(half) * top, got)
