"""Attention with a window: what a scale of zero makes of scores that are not finite."""
import math

import pytest
import torch

import paper_2411_03357_amd as pgcm
import kv_reference as ref16
import kv_window_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("half", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.0, -0.0, 0.25, -0.25])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_queries_that_are_not_finite(dim, scale, half):
    """zero times infinity is no number: alone and among many rows, and no other row changes"""
    for news in ([1, 1], [40, 7]):
        b = ref.Blocks(1, [90, 33], 2, dim, half)
        q = ref16.numbers(2, sum(news), 8, dim).to(half)
        clean, clean_lse = ref.run(pgcm, b, q, news, 30, 4, scale=scale)
        bad = torch.zeros(sum(news), 8, dtype=torch.bool, device="cuda")
        for row, head, channel, x in ((0, 3, 5, math.nan), (0, 6, dim - 1, math.nan), (sum(news) - 1, 1, 9, math.inf),
                                      (sum(news) - 1, 2, 0, -math.inf)):
            if scale != 0.0 and not math.isnan(x):
                continue    # (scores of minus infinity have no weight)
            q[row, head, channel] = x
            bad[row, head] = True
        out, lse = ref.run(pgcm, b, q, news, 30, 4, scale=scale)
        assert bool(torch.isnan(out[bad]).all()) and bool(torch.isnan(lse[bad]).all())
        assert torch.equal(out[~bad], clean[~bad]) and torch.equal(lse[~bad], clean_lse[~bad])
        if scale == 0.0:
            ref.check(pgcm, b, ref16.numbers(3, sum(news), 8, dim).to(half), news, 30, 4, scale=scale)
