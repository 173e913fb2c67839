"""The step that evens out what experts get."""
import pytest
import torch

import paper_2505_15511_amd as nomad
from test_gpu_map_operators import note

pytestmark = pytest.mark.gpu


def test_loads_come_to_the_mean():
    """Logits that favour one expert, and loads that come to the mean and stay there.

    A step moves an expert's sums by `rate` and those that they are compared with by as much the other way, so that of n rows at most n times 2 rate times the largest
    density of a score change sides: of 1 / (1 + e^-x) that is phi(x - 2) / (s (1 - s)) <= 5.4 for normal logits about 2 (at x = 2.9; 1.6 about 0). With 4,096 rows and the last
    rate of 5e-4 these are 22 rows on average, and with five deviations of such a count 47. The way there: sums differ by less than 1, 200 steps of 5e-3."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(4096, 16, device="cuda", generator=gen)
    logits[:, 3] += 2.0
    bias = torch.zeros(16, device="cuda")
    loads = lambda: torch.diff(nomad.route_scored(logits, 2, bias=bias).offsets)   # noqa: E731
    first = loads()
    assert first.max().item() > 2 * 512
    for rate, steps in ((5e-3, 200), (5e-4, 100)):
        for _ in range(steps):
            bias = nomad.balance_bias(bias, nomad.route_scored(logits, 2, bias=bias).offsets, rate)
    off = (loads() - 512).abs().max().item()
    note(f"  largest load {first.max().item()}, then {off} off the mean of 512")
    assert off <= 47


@pytest.mark.parametrize("rate", [1e39, -1e39, float("inf"), float("nan")])
def test_rates_that_are_no_float32_number(rate):
    offsets = nomad.route_scored(torch.zeros(10, 12, device="cuda"), 2).offsets
    with pytest.raises(ValueError):
        nomad.balance_bias(torch.zeros(12, device="cuda"), offsets, rate)
