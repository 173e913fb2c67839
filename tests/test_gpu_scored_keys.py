"""Routing by scores where sums lie so near each other, or so near the smallest bias, that 32 bits hardly tell them apart: rows of up to 256 experts, whose keys
sixteen lanes hold (tests/test_scored_keys.py goes through the same on the CPU)."""
import math

import numpy as np
import pytest
import torch

import paper_2505_15511_amd as nomad
from oracle import map_oracle as mo
from test_gpu_more_operators import check_scored
from test_gpu_map_operators import BF16, F16, F32, host, note

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


def repeated(rng, n, experts, value):
    """Rows of one logit, some of them moved by a few units, some far below."""
    x = np.full((n, experts), value, np.float32)
    moved = rng.random(x.shape) < np.array([0.0, 0.02, 0.1, 0.5])[rng.integers(0, 4, n)][:, None]
    x = np.where(moved, x.view(np.int32) + rng.integers(-200, 201, x.shape), x.view(np.int32)).astype(np.int32).view(np.float32)
    return np.where(rng.random(x.shape) < np.array([0.0, 0.5, 0.9])[rng.integers(0, 3, n)][:, None], value - 5.0, x)


@pytest.mark.parametrize("experts,dtype", [(50, F32), (64, BF16), (128, F32), (200, F32), (200, F16), (256, F32), (256, BF16), (256, F16)])
@pytest.mark.parametrize("biased", ["no", "zero", "two"])
def test_logits_that_are_the_same_but_for_a_few(experts, dtype, biased):
    """More equal sums in one lane than it keeps, and larger ones among those that it lets go."""
    note(f"repeated {experts} {dtype} {biased}")
    rng = np.random.default_rng(experts + len(biased))
    x = np.concatenate([repeated(rng, 60, experts, v) for v in (1.0, 6.0, 17.0, -9.0)] + [rng.integers(-3, 4, (60, experts)) * 7.0])
    x[::9, experts // 3:] = -math.inf
    logits = torch.from_numpy(x).to("cuda", dtype)
    bias = {"no": None, "zero": torch.zeros(experts, device="cuda"), "two": 0.25 * (torch.arange(experts, device="cuda") % 2)}[biased]
    for score in ("sigmoid", "softmax"):
        for k, more in ((1, {}), (2, {}), (3, {}), (8, {}), (2, dict(groups=2, top_groups=1)), (8, dict(groups=4, top_groups=2, group_best=2)), (8, dict(groups=8, top_groups=3))):
            if experts % more.get("groups", 1):
                continue
            r = nomad.route_scored(logits.repeat(8, 1), k, bias=bias, score=score, **more)
            want, weights = mo.route_scored(host(logits), k, bias=None if bias is None else bias.cpu().numpy(), score=score, **more)[:2]
            assert np.array_equal(r.experts.cpu().numpy(), np.tile(want, (8, 1))), (score, k, more)
            assert np.abs(host(r.weights) - np.tile(weights, (8, 1))).max() <= 2.0 ** -18   # (at most 1, good to a few tens of units of 2^-24)
            assert torch.equal(torch.diff(r.offsets), torch.bincount(r.experts[r.experts >= 0], minlength=experts).int())


def test_the_best_of_a_lane_s_equals():
    """Four or eight equal logits in one lane, and one in it that is larger by less than a key holds."""
    note("best of equals")
    up = float(np.nextafter(np.float32(6.0), np.float32(7.0)))
    for experts, equal, value, at, larger, rest, dtype, k, bias, want in (
            (128, (0, 1, 2, 3), 1.0, 64, 1 + 2.0 ** -18, 0.0, F32, 1, False, [64]), (128, (0, 1, 2, 3), 1.0, 64, 1 + 2.0 ** -18, 0.0, F32, 2, False, [64, 0]),
            (64, (0, 1, 2, 3), 20.0, 4, 21.0, 0.0, BF16, 2, True, [4, 0]), (128, (0, 1, 2, 3), 6.0, 64, up, 0.0, F32, 1, True, [64]),
            (256, (0, 1, 2, 3, 64, 65, 66, 67), 1.0, 128, 1 + 2.0 ** -18, 0.0, F32, 3, False, [128, 0, 1])):
        x = torch.full((1500, experts), rest, device="cuda", dtype=dtype)
        x[:, list(equal)] = value
        x[:, at] = larger
        zero = torch.zeros(experts, device="cuda") if bias else None
        assert nomad.route_scored(x, k, bias=zero).experts.unique(dim=0).tolist() == [want]
        if not bias:
            assert nomad.route(x, k).experts.unique(dim=0).tolist() == [want]
