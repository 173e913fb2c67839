"""Routing by scores where sums lie so near each other, or so near the smallest bias, that 32 bits hardly tell them apart: rows of up to 256 experts, whose keys
sixteen lanes hold (tests/test_scored_keys.py goes through the same on the CPU)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_more_operators import check_scored
from test_gpu_map_operators import BF16, F16, F32, note

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("experts,dtype", [(50, F16), (64, F32), (160, BF16), (160, F32), (200, F16), (256, F32)])
@pytest.mark.parametrize("score,spread,low", [("softmax", 6.0, 0.0), ("softmax", 30.0, 0.0), ("sigmoid", 1.0, -18.0), ("sigmoid", 0.2, -14.0)])
def test_scores_that_are_all_but_zero(experts, dtype, score, spread, low):
    """With a bias of zero, as a fit that evens out its experts begins: what the last places go to is hardly more than nothing."""
    note(f"all but zero {experts} {dtype} {score} {spread}")
    rng = np.random.default_rng(experts)
    n = 33_000 // experts + 300                                           # more than one workgroup does by itself
    x = spread * rng.normal(size=(n, experts)) + low
    x[::7, 1:] = -math.inf
    logits = torch.from_numpy(x).to("cuda", dtype)
    zero = torch.zeros(experts, device="cuda")
    for k in (1, 2, 3, 8):
        check_scored(logits, k, zero, score=score)
        if experts % 4 == 0:
            check_scored(logits, k, zero, score=score, groups=4, top_groups=2, group_best=2)
