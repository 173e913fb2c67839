"""What fitting a placer takes of the GPU's memory."""
import pytest
import torch

from paper_2505_15511_amd import placement

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_fit_holds_no_logits_of_all_rows(score):
    """300,000 rows and 2,048 clusters: 2.5 GB of logits, where the vectors are 10 MB; 65,536 rows of them, twice, are 1.1 GB."""
    n, d, clusters = 300_000, 8, 2048
    gen = torch.Generator(device="cuda").manual_seed(5)
    centres = 10.0 * torch.randn(clusters, d, device="cuda", generator=gen)
    labels = torch.randint(0, clusters, (n,), device="cuda", generator=gen)
    X = centres[labels] + torch.randn(n, d, device="cuda", generator=gen)
    theta = X[:, :2].contiguous()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    placer = placement.Placer.fit(X, theta, labels, clusters, hidden=8, epochs=0, score=score)
    assert torch.cuda.max_memory_allocated() - before < 1.5e9
    if score == "sigmoid":   # the nearest centre's logit is about zero on the average of all rows
        top = torch.cat([(placer._inputs(x) @ placer.router.t() + placer.router_bias).amax(1) for x in X.split(50_000)])
        assert abs(top.double().mean().item()) < 1e-3 * top.double().std().item()
