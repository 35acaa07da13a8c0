"""What the header of the operators on KV blocks says of the numbers that they are defined by."""
import numpy as np
import pytest
import torch

import kv_reference as ref


@pytest.mark.parametrize("half", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,tokens,std", [(64, 1, 1.0), (128, 16, 1.0), (8, 3, 20.0), (256, 64, 1e-3)])
def test_how_far_a_score_is_from_a_bound(half, dim, tokens, std):
    """q . k is more than a block's score at times, and never more than the score with half a step for what each of its factors
    may have been rounded by"""
    n, heads = 200, 4
    k = ref.numbers(dim, n, tokens, 1, dim, std=std).to(half)
    q = ref.numbers(dim + 1, 1, heads, dim).to(half)
    bounds, scales = ref.summarize(k, [tokens] * n)
    low, high = bounds[:, None, 0, 0], bounds[:, None, 0, 1]
    c, s = ref.eighths(q.float().numpy())
    c = c[0][None]
    step = scales.astype(np.float64) * s[0].astype(np.float64)
    best = np.maximum(c * low, c * high).sum(-1)
    largest = torch.einsum("hd,ntd->nht", q[0].double(), k[:, :, 0].double()).amax(-1).numpy()
    slack = ((np.abs(c) + np.maximum(np.abs(low), np.abs(high))) / 2 + 0.25).sum(-1)
    assert (largest <= (best + slack) * step * (1 + 2.0 ** -20)).all()
    if tokens == 1:
        assert (largest > best * step).any()
