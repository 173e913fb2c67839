"""The learned map as a user has it: fitted to a projection, it places vectors that it has not seen next to their like."""
import pytest
import torch

from paper_2505_15511_amd import pipeline, placement, workloads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_fitted_map_places_new_vectors(bits):
    print(f"placement bits={bits}", flush=True)
    X, _ = workloads.gmm_points(6000, 50, 10, 25.0, 7, mix="equal", interleave=True)
    X = X.cuda()
    seen, new = X[:5000].contiguous(), X[5000:].contiguous()
    theta, info = pipeline.project(seen, 10, k=15, n_epochs=100, return_info=True)
    placer, losses = placement.Placer.fit(seen, theta, info["labels"], info["n_clusters"], hidden=64, epochs=30, batch=1024, bits=bits, return_losses=True)
    first, last = losses[:5].mean().item(), losses[-5:].mean().item()
    print(f"  loss {first:.4f} -> {last:.4f}", flush=True)
    assert last < 0.1 * first
    places = placer(new)
    assert places.shape == (1000, 2) and torch.isfinite(places).all()
    # the nearest seen neighbour of a new vector stands near the place it was given: nearer than a random point in most cases
    nearest = torch.cdist(new, seen).argmin(1)
    off = (places - theta[nearest]).norm(dim=1)
    chance = (places - theta[torch.randperm(5000, device="cuda")[:1000]]).norm(dim=1)
    assert off.median() < 0.15 * chance.median()
    one = placer(new[3:4])                                     # a single vector, as in serving
    assert (one - places[3:4]).abs().max() < 1e-4 * placer.spread


def test_step_moves_against_the_gradient_of_the_loss():
    """The step's gradients against differences of the loss that it returns.  Every expert is chosen: the loss jumps where
    a shift of the router changes the choice."""
    print("placement gradients", flush=True)
    torch.manual_seed(5)
    x, target = torch.randn(40, 9, device="cuda"), torch.randn(40, 2, device="cuda")
    p = placement.Placer(9, 4, hidden=6, k=4, seed=3)
    before = [t.clone() for t in p.parameters()]
    m = [torch.zeros_like(t) for t in before]

    def loss():
        y = p(x)
        return (y - target).pow(2).sum(1).mean().double().item()
    p._states = [(a, torch.zeros_like(a)) for a in m]
    p.step(x, target, lr=0.0)
    for t, b, a, name in zip(p.parameters(), before, m, p.NAMES):
        assert torch.equal(t, b)                               # a rate of zero: only the averages have moved, by a tenth of the gradient
        g = 10.0 * a
        for at in torch.randperm(t.numel())[:6].tolist():
            flat, h = t.view(-1), 2e-2 if name.startswith("router") else 5e-2
            old = flat[at].item()
            flat[at] = old + h
            up = loss()
            flat[at] = old - h
            down = loss()
            flat[at] = old
            got, want = g.view(-1)[at].item(), (up - down) / (2 * h)
            assert abs(got - want) < 2e-2 * (abs(want) + g.abs().max().item()) + 1e-3, (name, at, got, want)
