"""Attention with a window: a new token's results are as near to the definition among many as alone.

Values follow each other in pairs of opposite signs under nearly equal weights, so that an output is a hundredth of the sum of its
parts' sizes or less: its own rounding does not hide what its weights have lost."""
import math

import numpy as np
import pytest
import torch

import paper_2411_03357_amd as pgcm
import kv_reference as ref16
import kv_window_reference as ref

pytestmark = pytest.mark.gpu

# of a weight in [1, 2), what its two halves leave out: the first, towards zero, less than its last bit (2^-10; 2^-7), and the second,
# to nearest, half of the last bit of a number below that (2^-22; 2^-16)
LEFT_OUT = {torch.float16: 2.0 ** -22, torch.bfloat16: 2.0 ** -16}
SCALE = 0.125


def _whole(seed, shape, most, by):
    return torch.from_numpy(np.random.default_rng([83, seed]).integers(-most, most + 1, shape)).double() / by


def _setup(half, kv, group, dim, length, new):
    """keys and queries are eighths and halves of whole numbers: scores are exact in 32 bits, in any order"""
    b = ref.Blocks(1, [length], kv, dim, half)
    k, v = _whole(2, (length, kv, dim), 8, 8), ref16.numbers(3, length, kv, dim).to(half).double()
    k[1::2] = k[:-1:2][:k[1::2].shape[0]]
    k[1::2, :, dim // 2] += 0.125
    v[1::2] = -v[:-1:2][:v[1::2].shape[0]]
    for to, of in ((b.r.k, k), (b.r.v, v)):
        for t in range(length):
            to[int(b.tables[0, t // 16]), t % 16] = of[t].to(half)
    return b, k, v, _whole(4, (new, kv * group, dim), 2, 2)


def _bounds(half, q, k, v, window, sinks):
    """out in 64 bits, and how far it may be off: its rounding; n additions of weights and of their products; the exponential and its
    argument, 2^-22 of the largest; and what the halves of a weight leave out, or 2^-38 of the largest in binary16"""
    new, heads, dim = q.shape
    length, kv, _ = k.shape
    group = heads // kv
    out, tol = torch.zeros(new, heads, dim, dtype=torch.float64), torch.zeros(new, heads, dim, dtype=torch.float64)
    for j in range(new):
        end = length - (new - 1 - j)
        seen = torch.tensor([t for t in range(end) if window == 0 or t >= end - window or t < sinks])
        for h in range(heads):
            kh, vh = k[seen, h // group], v[seen, h // group]
            s = (kh @ q[j, h]) * SCALE
            p = torch.softmax(s, 0)
            size = p @ vh.abs()
            off = 2 * len(seen) * 2.0 ** -24 + 2.0 ** -22 * (1.5 * float(s.abs().max()) + 4) + LEFT_OUT[half]
            out[j, h] = p @ vh
            tol[j, h] = ref16.UNIT[half] * out[j, h].abs() + ref16.LEAST[half] + 1.01 * off * size
            if half == torch.float16:
                tol[j, h] += 2.0 ** -38 * p.max() * vh.abs().sum(0)
    return out, tol


@pytest.mark.parametrize("half", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kv, group, dim, length, new, window, sinks", [
    (2, 4, 128, 100, 40, 0, 0), (1, 3, 64, 90, 50, 48, 6), (1, 2, 256, 70, 33, 0, 0), (3, 1, 80, 101, 101, 64, 4), (1, 130, 24, 64, 2, 0, 0)])
def test_weights_keep_their_bits_among_many_rows(half, kv, group, dim, length, new, window, sinks):
    b, k, v, q = _setup(half, kv, group, dim, length, new)
    want, tol = _bounds(half, q, k, v, window, sinks)
    out, _ = ref.run(pgcm, b, q.to(half), [new], window, sinks, scale=SCALE)
    ref16.within(out, (want, tol), "out")
    # the last one alone
    out, _ = ref.run(pgcm, b, q[-1:].to(half), [1], window, sinks, scale=SCALE)
    ref16.within(out, (want[-1:], tol[-1:]), "out alone")
    assert math.isfinite(float(out.float().sum()))
