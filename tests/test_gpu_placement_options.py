"""The learned map with routing by scores, groups, balance, a shared expert and a limit on its gradients' norm."""
import math

import pytest
import torch

from paper_2505_15511_amd import placement
from test_gpu_placement import _projected

pytestmark = pytest.mark.gpu

OPTIONS = [dict(score="sigmoid"), dict(balance=1e-3), dict(shared=48), dict(max_norm=0.05), dict(groups=None, top_groups=2, group_best=2),
           dict(score="sigmoid", groups=None, top_groups=2, balance=1e-3, shared=33, max_norm=0.1)]


def _of(options, n_clusters):
    """groups: as few as the clusters that are left can be cut into."""
    return {name: next(g for g in range(2, n_clusters + 1) if n_clusters % g == 0) if name == "groups" else value for name, value in options.items()}


@pytest.mark.parametrize("options", OPTIONS, ids=lambda o: "-".join(o))
def test_fits(options):
    """It runs, twice alike, with finite places for new vectors, one by one as together."""
    print(f"placement {options}", flush=True)
    seen, new, theta, info = _projected(3000)
    options = _of(options, info["n_clusters"])
    fits = [placement.Placer.fit(seen, theta, info["labels"], info["n_clusters"], hidden=32, epochs=2, batch=700, **options) for _ in range(2)]
    assert all(torch.equal(a, b) for a, b in zip(fits[0].parameters(), fits[1].parameters()))
    places = fits[0](new)
    assert places.shape == (1000, 2) and torch.isfinite(places).all() and torch.equal(places, fits[1](new))
    assert (fits[0](new[3:4]) - places[3:4]).abs().max() < 1e-4 * fits[0].spread
    if "max_norm" in options:
        assert fits[0].norm.shape == (1,) and math.isfinite(fits[0].norm.item())
    if "balance" in options:
        assert fits[0].balance_bias.abs().max() > 0


def _loss(placer, x, target):
    """The step's loss in 64 bits, experts as they are chosen now; the placer's parameters as leaves."""
    p = {name: getattr(placer, name).double().requires_grad_() for name in placer.names}
    xx = ((x - placer.shift) * placer.scale).double()
    logits = xx @ p["router"].t() + p["router_bias"]
    chosen = placer._route(placer._logits(placer._inputs(x), placer._one(x.shape[0]))).experts.long()
    s = torch.sigmoid(logits) if placer.scoring["score"] == "sigmoid" else torch.softmax(logits, 1)
    picked = s.gather(1, chosen)
    weights = picked / picked.sum(1, keepdim=True)
    h = torch.nn.functional.silu(torch.matmul(p["w1"][chosen], xx[:, None, :, None])[..., 0] + p["b1"][chosen])
    y = (weights[..., None] * (torch.matmul(p["w2"][chosen], h[..., None])[..., 0] + p["b2"][chosen])).sum(1)
    if "s1" in p:
        y = y + torch.nn.functional.silu(xx @ p["s1"].t() + p["t1"]) @ p["s2"].t() + p["t2"]
    return ((y - (target / placer.spread).double()) ** 2).sum(1).mean(), p


@pytest.mark.parametrize("options", OPTIONS, ids=lambda o: "-".join(o))
def test_a_step_is_adamw_on_its_gradients(options):
    """The first step of AdamW without decay moves a parameter by lr g / (|g| + eps): where a gradient in 64 bits is well above its rounding, by
    its sign; the returned loss is the one in 64 bits."""
    seen, _, theta, info = _projected(2000)
    options = _of(options, info["n_clusters"])
    placer = placement.Placer.fit(seen, theta, info["labels"], info["n_clusters"], hidden=32, epochs=0, **options)
    x, target = seen[:512], theta[:512]
    loss, leaves = _loss(placer, x, target)
    loss.backward()
    before = [p.clone() for p in placer.parameters()]
    got = placer.step(x, target, lr=1e-3)
    assert abs(got.item() - loss.item()) < 1e-4 * loss.item()
    grads = [leaves[name].grad for name in placer.names]
    norm = math.sqrt(sum(float((g * g).sum()) for g in grads))
    if placer.max_norm is not None:
        assert abs(placer.norm.item() - norm) < 1e-3 * norm
    for name, p, old, g in zip(placer.names, placer.parameters(), before, grads):
        # eps is 1e-8 and clipping makes gradients smaller: what moved by nearly lr has a gradient far above eps
        clear = g.abs() > 1e-3 * g.abs().max() + 1e-6
        moved = (old - p).double()
        assert torch.equal(torch.sign(moved[clear]), torch.sign(g[clear])), name


def test_refusals():
    bad = [dict(groups=3), dict(groups=2, top_groups=3), dict(groups=10, top_groups=1), dict(score="tanh"), dict(balance=-1.0), dict(max_norm=-1.0), dict(shared=-1), dict(groups=0)]
    for options in bad:
        with pytest.raises(ValueError):
            placement.Placer(8, 10, **options)
