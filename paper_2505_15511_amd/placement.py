"""A learned map: a function that places vectors on a finished projection, also those that it was not made from.

`pipeline.project` ends with a table of points; a new vector has no row in it.  Here every cluster of the partition has an
expert, a small network of two layers that has learned its region; a router, linear in the vector, chooses the experts that
answer and weighs them, so that the map is continuous across borders; the step that fits them is AdamW.  Router, products, sums over
experts and clusters, gradients, their norm and the step are the library's operators; scaling, the residual and the rows of a batch are torch's.

Maps of many clusters have more to choose from: sigmoid scores, groups of neighbouring clusters of which a vector asks a few, a bias that
evens out how many vectors an expert gets (`balance`), an expert that all vectors share (`shared`), and steps whose gradients' norm is
limited (`max_norm`).

    theta, info = pipeline.project(X, n_clusters=256, return_info=True)
    placer = placement.Placer.fit(X, theta, info["labels"], info["n_clusters"])
    new_points = placer(new_vectors)                                    # [m, 2]
"""
from __future__ import annotations

import torch

from .operators import (adamw_state, adamw_step, balance_bias, combine, combine_gradient, dense_gradient, dense_product, gradient_norm, grouped_product,
                        grouped_weight_gradient, route, route_gradient, route_scored, route_scored_gradient)


def experts(x, routing, w1, b1, w2, b2, activation="silu", keep=False):
    """The rows' experts, weighed: y_i = sum_j weights_ij (act(x_i W1^T + b1) W2^T + b2) of the routing's experts.  x [n, d],
    w1 [E, h, d], w2 [E, o, h]; keep=True returns (y, what `experts_gradient` takes)."""
    per_row = routing.slots.shape[1]
    hidden = grouped_product(x, w1, routing.offsets, b1, activation, order=routing.order, per_row=per_row, keep=keep)
    h, z = hidden if keep else (hidden, None)
    o = grouped_product(h, w2, routing.offsets, b2)
    y = combine(o, routing.slots, routing.weights)
    return (y, (z, h, o)) if keep else y


def experts_gradient(dy, x, routing, w1, b1, w2, b2, kept, activation="silu", need_dx=True):
    """The gradients of `experts` from dy [n, o]: dict(dx, dweights, dw1, db1, dw2, db2); weights' in their own type, the
    biases' and dweights in float32."""
    z, h, o = kept
    per_row = routing.slots.shape[1]
    do, dweights = combine_gradient(dy, o, routing.slots, routing.weights, order=routing.order)
    dw2, db2 = grouped_weight_gradient(do, h, routing.offsets)
    dz = grouped_product(do, w2.transpose(1, 2), routing.offsets, activation=activation, slope_at=z)
    dw1, db1 = grouped_weight_gradient(dz, x, routing.offsets, order=routing.order, per_row=per_row)
    dx = combine(grouped_product(dz, w1.transpose(1, 2), routing.offsets), routing.slots) if need_dx else None
    return {"dx": dx, "dweights": dweights, "dw1": dw1, "db1": db1, "dw2": dw2, "db2": db2}


class Placer:
    """Router and experts of a map, and the step that fits them.

    Inputs are centred and scaled, and the plane scaled, as the data says (`shift`, `scale`, `spread`).  Parameters are float32:
    router [E, d] with bias [E], w1 [E, h, d], b1 [E, h], w2 [E, 2, h], b2 [E, 2], and of the shared expert of `shared` columns s1 [shared, d],
    t1 [shared], s2 [2, shared], t2 [2].

    score: of the router's logits, "softmax" or "sigmoid"; groups, top_groups, group_best: as `route_scored` takes them; balance: the step, every
    fitting step, of a bias on the scores that the choice is made by (0: none); max_norm: what a step's gradients are scaled down to
    (None: they are not)."""

    NAMES = ("router", "router_bias", "w1", "b1", "w2", "b2")
    SHARED_NAMES = ("s1", "t1", "s2", "t2")

    def __init__(self, d, n_experts, hidden=128, k=2, out=2, bits=32, seed=0, device="cuda", score="softmax", groups=1, top_groups=1, group_best=1, balance=0.0, shared=0, max_norm=None):
        if not (1 <= k <= n_experts and hidden >= 1 and d >= 1 and out >= 1 and shared >= 0):
            raise ValueError("1 <= k <= n_experts, and at least one column everywhere")
        if groups < 1 or n_experts % groups or not 1 <= top_groups <= groups or k > top_groups * (n_experts // groups):
            raise ValueError(f"{n_experts} experts in {groups} groups, {top_groups} of them open, have no room for k = {k}")
        if score not in ("softmax", "sigmoid") or not balance >= 0.0 or (max_norm is not None and not max_norm >= 0.0):
            raise ValueError("score is softmax or sigmoid, balance and max_norm are not negative")
        gen = torch.Generator().manual_seed(seed)
        draw = lambda *shape, scale: (scale * torch.randn(*shape, generator=gen)).to(device)   # noqa: E731
        self.k, self.bits, self.steps = int(k), bits, 0
        self.router, self.router_bias = draw(n_experts, d, scale=d ** -0.5), torch.zeros(n_experts, device=device)
        self.w1, self.b1 = draw(n_experts, hidden, d, scale=d ** -0.5), torch.zeros(n_experts, hidden, device=device)
        self.w2, self.b2 = draw(n_experts, out, hidden, scale=hidden ** -0.5), torch.zeros(n_experts, out, device=device)
        self.shift, self.scale, self.spread = torch.zeros(d, device=device), torch.ones((), device=device), torch.ones((), device=device)
        self.scoring = {"score": score, "groups": groups, "top_groups": top_groups, "group_best": group_best}
        self.balance, self.max_norm, self.norm = float(balance), max_norm, None
        self.balance_bias = torch.zeros(n_experts, device=device) if balance else None
        if shared:
            self.s1, self.t1 = draw(shared, d, scale=d ** -0.5), torch.zeros(shared, device=device)
            self.s2, self.t2 = draw(out, shared, scale=shared ** -0.5), torch.zeros(out, device=device)
        self.names = self.NAMES + (self.SHARED_NAMES if shared else ())
        self._states = [adamw_state(p, bits) for p in self.parameters()]

    def parameters(self):
        return [getattr(self, name) for name in self.names]

    def _one(self, n):
        """Offsets of a single group of n rows: the router is a product with one group."""
        return torch.arange(2, dtype=torch.int32, device=self.router.device) * n

    def _inputs(self, x):
        if x.dim() != 2 or x.shape[1] != self.shift.shape[0]:
            raise ValueError(f"vectors must be rows of {self.shift.shape[0]} columns, got shape {tuple(x.shape)}")
        return ((x.float() - self.shift) * self.scale).contiguous()

    def _logits(self, x, one):
        return grouped_product(x, self.router[None], one, self.router_bias[None])

    def _plain(self):
        """Whether the router's weights are a softmax over the k largest logits and nothing else."""
        return self.scoring["score"] == "softmax" and self.scoring["groups"] == 1 and self.balance_bias is None

    def _route(self, logits):
        return route(logits, self.k) if self._plain() else route_scored(logits, self.k, bias=self.balance_bias, **self.scoring)

    def __call__(self, x):
        """The places [m, 2] of the vectors x [m, d]."""
        x = self._inputs(x)
        routing = self._route(self._logits(x, self._one(x.shape[0])))
        y = experts(x, routing, self.w1, self.b1, self.w2, self.b2)
        if "s1" in self.names:
            y = dense_product(dense_product(x, self.s1, self.t1, "silu"), self.s2, self.t2, residual=y)
        return y * self.spread

    def step(self, x, target, lr=1e-3, weight_decay=0.0):
        """One AdamW step on the mean squared distance between the places of x and target [m, 2]; returns that distance (a
        tensor on the GPU, in units of the plane's spread, before the step).  With max_norm, `norm` is then the gradients' norm."""
        if not x.shape[0] or tuple(target.shape) != (x.shape[0], self.b2.shape[1]):
            raise ValueError(f"a step takes vectors, and as many places of {self.b2.shape[1]} coordinates")
        x, one = self._inputs(x), self._one(x.shape[0])
        logits = self._logits(x, one)
        routing = self._route(logits)
        y, kept = experts(x, routing, self.w1, self.b1, self.w2, self.b2, keep=True)
        if "s1" in self.names:
            h, z = dense_product(x, self.s1, self.t1, "silu", keep=True)
            y = dense_product(h, self.s2, self.t2, residual=y)
        off = (y - target / self.spread).contiguous()
        dy = off * (2.0 / x.shape[0])
        g = experts_gradient(dy, x, routing, self.w1, self.b1, self.w2, self.b2, kept, need_dx=False)
        if self._plain():
            dlogits = route_gradient(logits, routing, g["dweights"])
        else:
            dlogits = route_scored_gradient(logits, routing, g["dweights"], score=self.scoring["score"])
        drouter, drouter_bias = grouped_weight_gradient(dlogits, x, one)
        grads = [drouter, drouter_bias, g["dw1"], g["db1"], g["dw2"], g["db2"]]
        if "s1" in self.names:
            dh, ds2, dt2 = dense_gradient(dy, h, self.s2)
            _, ds1, dt1 = dense_gradient(dh, x, self.s1, "silu", z, need_dx=False)
            grads += [ds1, dt1, ds2, dt2]
        scale = None
        if self.max_norm is not None:
            self.norm, scale = gradient_norm(grads, self.max_norm)
        self.steps += 1
        adamw_step(self.parameters(), grads, [s[0] for s in self._states], [s[1] for s in self._states], self.steps, lr=lr, weight_decay=weight_decay,
                   grad_scale=scale, dither=self.bits == 8)
        if self.balance_bias is not None:
            self.balance_bias = balance_bias(self.balance_bias, routing.offsets, self.balance)
        return (off * off).sum(1).mean()

    @classmethod
    def fit(cls, X, theta, labels, n_clusters, hidden=128, k=2, epochs=10, batch=8192, lr=2e-3, bits=32, seed=0, return_losses=False, **more):
        """A placer that has learned the projection theta [n, 2] of X [n, d] (float32, on the GPU) with the partition `labels`.
        The router starts from the clusters' centres (the nearest centre has the largest logit), the experts' last biases
        from the clusters' places; the rate falls linearly to zero.  Two fits with the same arguments give the same map.  more: score, groups,
        top_groups, group_best, balance, shared and max_norm, as `Placer` takes them."""
        n, d = X.shape
        at = labels.long()
        low, high = (int(v) for v in at.aminmax()) if at.numel() else (0, 0)
        if tuple(at.shape) != (n,) or low < 0 or high >= n_clusters:
            raise ValueError(f"labels must be {n} whole numbers in 0..{n_clusters - 1}")
        placer = cls(d, n_clusters, hidden, min(k, n_clusters), 2, bits, seed, X.device, **more)
        # sums over clusters: the gradient of weights of one column out, in an order that does not depend on timing
        sizes, members = torch.bincount(at, minlength=n_clusters), torch.sort(at, stable=True).indices.int()
        count, ends = sizes.clamp(min=1).float()[:, None], torch.nn.functional.pad(sizes.cumsum(0), (1, 0)).int()
        ones = torch.ones(n, 1, device=X.device)

        def sums(values):
            return grouped_weight_gradient(ones, values.contiguous(), ends, order=members, bias=False)[0][:, 0]
        placer.shift = X.mean(0)
        placer.scale = 1.0 / (X - placer.shift).pow(2).mean().sqrt().clamp(min=1e-30)
        placer.spread = theta.pow(2).mean().sqrt().clamp(min=1e-30)
        centres = sums(placer._inputs(X)) / count
        # -|x - c|^2 / 2 without what all experts have in common, in units of the squared distance to a row's own centre
        width = (placer._inputs(X) - centres[at]).pow(2).sum(1).mean().clamp(min=1e-30)
        placer.router.copy_(centres * (4.0 / width))
        placer.router_bias.copy_(centres.pow(2).sum(1) * (-2.0 / width))
        if placer.scoring["score"] == "sigmoid":   # logits of the nearest centres about zero, where scores differ
            nearest = [(placer._inputs(rows) @ placer.router.t() + placer.router_bias).amax(1) for rows in X.split(1 << 16)]   # (never those of all rows at once)
            placer.router_bias -= torch.cat(nearest).mean()
        placer.b2.copy_(sums(theta / placer.spread) / count)
        gen = torch.Generator(device=X.device).manual_seed(seed)
        per, losses = max(1, -(-n // batch)), []
        for epoch in range(epochs):
            order = torch.randperm(n, generator=gen, device=X.device)
            for i in range(per):
                rows = order[i * batch:(i + 1) * batch]
                losses.append(placer.step(X[rows], theta[rows], lr * (1.0 - (epoch * per + i) / (epochs * per))))
        return (placer, torch.stack(losses)) if return_losses else placer
