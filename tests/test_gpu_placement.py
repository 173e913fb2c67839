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


def _projected(n=5000):
    X, _ = workloads.gmm_points(n + 1000, 50, 10, 25.0, 7, mix="equal", interleave=True)
    X = X.cuda()
    seen, new = X[:n].contiguous(), X[n:].contiguous()
    theta, info = pipeline.project(seen, 10, k=15, n_epochs=100, return_info=True)
    return seen, new, theta, info


def test_two_fits_of_one_seed_are_the_same_map():
    """Sums over clusters, like every operator's, do not depend on timing."""
    print("placement twice", flush=True)
    seen, new, theta, info = _projected()
    for bits in (32, 8):
        fits = [placement.Placer.fit(seen, theta, info["labels"], info["n_clusters"], hidden=32, epochs=2, batch=512, bits=bits) for _ in range(3)]
        for other in fits[1:]:
            assert all(torch.equal(a, b) for a, b in zip(fits[0].parameters(), other.parameters()))
            assert torch.equal(fits[0](new), other(new))


def test_the_start_is_made_of_the_clusters():
    """Without a step: centres and places of the clusters, against sums in 64 bits (a float32 sum of n terms is off by n + 8 units of 2^-24
    of their absolute sum, and what is made of it by a few more)."""
    print("placement start", flush=True)
    seen, new, theta, info = _projected()
    labels, groups = info["labels"].long(), info["n_clusters"]
    p = placement.Placer.fit(seen, theta, labels, groups, hidden=16, epochs=0)
    unit = (seen.shape[0] + 32) * 2.0 ** -24
    x, places = ((seen - p.shift) * p.scale).double(), (theta / p.spread).double()
    centres = torch.stack([x[labels == e].mean(0) for e in range(groups)])
    width = (x - centres[labels]).pow(2).sum(1).mean()
    size = torch.stack([x[labels == e].abs().mean(0) for e in range(groups)])
    assert ((p.router.double() - centres * (4.0 / width)).abs() <= 4 * unit * (4.0 / width) * (size + centres.abs())).all()
    want = torch.stack([places[labels == e].mean(0) for e in range(groups)])
    size = torch.stack([places[labels == e].abs().mean(0) for e in range(groups)])
    assert ((p.b2.double() - want).abs() <= 4 * unit * size).all()
    for bad in (labels + 1, labels[:-1]):
        with pytest.raises(ValueError):
            placement.Placer.fit(seen, theta, bad, groups, epochs=0)


def test_fitting_betters_the_start():
    """The start places a vector at its clusters' places; a fitted map places it nearer to its neighbour than that."""
    print("placement against its start", flush=True)
    seen, new, theta, info = _projected()
    target = theta[torch.cdist(new, seen).argmin(1)]
    off = [(placement.Placer.fit(seen, theta, info["labels"], info["n_clusters"], hidden=64, epochs=epochs, batch=1024)(new) - target).norm(dim=1).median().item() for epochs in (0, 30)]
    print(f"  median distance: start {off[0]:.4f}, fitted {off[1]:.4f}", flush=True)
    assert off[1] < off[0]


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


def test_vectors_in_any_layout_and_number():
    print("placement layouts", flush=True)
    torch.manual_seed(6)
    p, x = placement.Placer(20, 5, hidden=16, k=2, seed=1), torch.randn(64, 20, device="cuda")
    want = p(x)
    wide = torch.randn(64, 33, device="cuda")
    wide[:, 5:25] = x
    for same in (x.t().contiguous().t(), wide[:, 5:25], x.double()):
        assert torch.equal(p(same), want)
    assert p(x[:0]).shape == (0, 2)
    target = torch.randn(64, 2, device="cuda")
    pair = [placement.Placer(20, 5, hidden=16, k=2, seed=1) for _ in range(2)]
    pair[0].step(x, target)
    pair[1].step(x.t().contiguous().t(), target.t().contiguous().t())
    assert all(torch.equal(a, b) for a, b in zip(pair[0].parameters(), pair[1].parameters()))
    for bad in ((x[:0], target[:0]), (x, target[:63]), (x, target[:, 0]), (x[:, :19], target)):
        with pytest.raises(ValueError):
            p.step(*bad)
    with pytest.raises(ValueError):
        p(x[:, :19])
