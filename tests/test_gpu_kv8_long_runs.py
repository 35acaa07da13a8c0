"""Appends to blocks in 8 bits with norms and rotation, in runs that are longer than what a wavefront holds: taken twice, a part at a
time, in several rounds of heads, from inside a block on."""
import pytest
import torch

import paper_2411_03357_amd as pgcm
import kv8_reference as ref
import kv_reference as ref16

pytestmark = pytest.mark.gpu

EPS = 1e-5
F16, BF16 = torch.float16, torch.bfloat16
CASES = [  # block tokens, kv heads, query heads, channels, rotated ones, adjacent, norms, first call's tokens, second's, type
    (64, 4, 8, 128, 128, False, True, 0, 300, BF16),
    (64, 4, 0, 128, 128, False, True, 63, 129, F16),
    (256, 3, 6, 128, 64, True, True, 37, 700, BF16),
    (256, 3, 3, 128, 128, False, False, 200, 500, F16),
    (256, 2, 2, 128, None, False, True, 90, 600, BF16),
    (48, 5, 5, 80, 48, False, True, 47, 400, F16),
    (4096, 3, 3, 64, 64, False, True, 100, 2500, BF16),
    (4096, 1, 2, 64, 32, True, False, 0, 5000, F16),
    (256, 2, 2, 256, 256, False, True, 1, 400, BF16),
    (512, 300, 300, 16, 16, False, True, 5, 700, BF16),
    (16, 300, 0, 16, 16, True, True, 3, 100, F16),
    (1024, 260, 0, 16, 16, False, False, 400, 700, F16),
    (128, 1, 16, 144, 144, True, True, 0, 1000, BF16)]


@pytest.mark.parametrize("code", ref.CODES)
@pytest.mark.parametrize("case", CASES)
def test_long_runs_with_norms_and_rotation(case, code):
    block, kv, heads, dim, rope_dim, adjacent, weighted, first, second, half = case
    n, places = first + second, 997
    blocks = -(-n // block)
    x = ref16.numbers(61, n, heads + 2 * kv, dim) * 2.0 ** ref16.numbers(62, n, heads + 2 * kv, 1, std=3.0).clamp(-9, 9)
    x = x.to(half)
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    weights = [(1 + 0.2 * ref16.numbers(63 + i, dim)).to(half) if weighted else None for i in (0, 1)]
    positions = [(7919 * t + t // 3) % places for t in range(n)]
    table = None
    if rope_dim is not None:
        angle = torch.arange(places).double()[:, None] * 100.0 ** (-torch.arange(0, rope_dim, 2).double() / rope_dim)
        table = torch.cat([angle.cos(), angle.sin()], 1).float()
    order = torch.randperm(blocks + 1, generator=torch.Generator().manual_seed(block + dim))
    at = torch.arange(n)
    slots = order[at // block] * block + at % block
    cpu = ref.pool8(64, blocks + 1, block, kv, dim, code)
    gpu = ref.on_gpu(cpu, block, kv, dim, code, True)
    cache8 = pgcm.KV8Cache(*gpu, half)
    on, at_gpu, slots_gpu = x.cuda(), torch.tensor(positions, dtype=torch.int32).cuda(), slots.cuda()
    q_out = torch.full((n, heads, dim), 7.0, dtype=half, device="cuda")
    for a, b in ((0, first), (first, n)):
        if a == b:
            continue
        pgcm.kv8_append(cache8, on[a:b, :heads] if heads else None, on[a:b, heads:heads + kv], on[a:b, heads + kv:],
                        None if table is None else at_gpu[a:b], slots_gpu[a:b], q_out[a:b] if heads else None,
                        q_weight=weights[0].cuda() if weighted and heads else None, k_weight=weights[1].cuda() if weighted else None,
                        eps=EPS, rope=None if table is None else table.cuda(), adjacent=adjacent)
    # sums of dim squares, their mean, root and quotient, the factors and two products: each a rounding of 2^-24 or two, of a pair's
    # larger part
    slack = 2 * (dim + 24) * 2.0 ** -24
    if heads:
        want = ref16.turned(q, weights[0], EPS, table, positions, adjacent)
        near = ref16.UNIT[half] * want.abs() + ref16.LEAST[half] + slack * want.abs().amax(-1, keepdim=True)
        ref16.within(q_out, (want, near), "q")
    want_k = ref16.turned(k, weights[1], EPS, table, positions, adjacent)
    for i, want in enumerate((want_k, v.double())):
        slack_of = 0.0 if i else slack
        scales = gpu[2 + i].cpu().double()[order[at // block]]                      # [token][head]
        codes = gpu[i].float().cpu().double()[order[at // block], at % block]
        # each block's scale is the least power of two that reaches its largest value
        rows = torch.zeros(blocks * block, kv, dtype=torch.float64)
        rows[:n] = want.abs().amax(-1)
        largest = rows.view(blocks, block, kv).amax(1)[at // block]
        assert bool((torch.frexp(scales).mantissa == 0.5).all())
        assert bool((ref.TOP[code] * scales >= largest * (1 - slack_of)).all()), "kv"[i]
        assert bool((ref.TOP[code] * scales / 2 < largest * (1 + slack_of)).all()), "kv"[i]
        # codes are the nearest; those that were there before the second call may have been rounded again
        again = ((at < first) & (at // block == first // block))[:, None, None]
        s = scales[..., None]
        if code == torch.int8:
            step = torch.where(again, s, s / 2)
        else:
            step = torch.maximum(want.abs() / 16, torch.where(again, s * 2.0 ** -9, s * 2.0 ** -10))
        off = (codes * s - want).abs()
        assert bool((off <= step * (1 + 2.0 ** -20) + slack_of * want.abs().amax(-1, keepdim=True)).all()), \
            ("kv"[i], (off - step).max(), torch.nonzero(off > step * 1.01 + slack_of * want.abs().amax(-1, keepdim=True))[:3].tolist())
        # the block that no token went to is as it was
        spare = order[blocks]
        assert torch.equal(gpu[i][spare].cpu().view(torch.uint8), cpu[i][spare].view(torch.uint8))
        assert torch.equal(gpu[2 + i][spare].cpu(), cpu[2 + i][spare])
