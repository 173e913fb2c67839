"""More operators of a learned map as measurable cases: routing by scores with a bias for balance and groups of experts, the
dense product with bias, activation and residual of an expert that all rows share, and the gradients' norm with the factor
that clips a step.

A router's inputs are as a map's fitting leaves them: logits about their expert's own level, a balancing bias of two hundredths, a row in 64
padding, whose logits are all -inf."""
import math

import torch

own = False          # whether run() makes the framework's calls; its package is imported where they are made

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BALANCE = 1e-3       # the step of the bias


def _routing(name, n, experts, k, **more):
    return {"name": name, "kind": "route", "n": n, "experts": experts, "k": k, **more}


def _dense(name, n, d, out, **more):
    return {"name": name, "kind": "dense", "n": n, "d": d, "out": out, **more}


def listed():
    return [
        # One vector asks for its regions of a map of 256 clusters in eight groups: the latency of a call.
        _routing("scored-1", 1, 256, 8, groups=8, top_groups=4, best=2, score="sigmoid", bias=True, normalize=True, scale=2.5, dtype="f32", gradient=False),
        # A pass of fitting over large batches: grouped experts, the logits' gradient and the bias' step.
        _routing("scored-300k-groups", 300_000, 256, 8, groups=8, top_groups=4, best=2, score="sigmoid", bias=True, normalize=True, scale=2.5, dtype="bf16", gradient=True),
        # The default partition's router with balance, no groups: two experts a row.
        _routing("scored-500k", 500_000, 256, 2, groups=1, top_groups=1, best=1, score="sigmoid", bias=True, normalize=True, scale=1.0, dtype="f32", gradient=True),
        # Softmax scores that keep their share of all experts, odd numbers of experts and rows.
        _routing("scored-odd", 40_037, 50, 3, groups=5, top_groups=2, best=1, score="softmax", bias=True, normalize=False, scale=1.0, dtype="f16", gradient=True),
        # A single vector through the shared expert's first layer.
        _dense("dense-1", 1, 768, 2048, dtype="bf16", activation="silu", residual=False, keep=False, turned=False, back=False),
        # A small batch of queries through a wide layer: the weights' bytes.
        _dense("dense-24", 24, 8192, 4096, dtype="f16", activation="none", residual=True, keep=False, turned=False, back=False),
        # Few tiles and a long sum: the units have to share it.
        _dense("dense-500-long", 500, 8192, 768, dtype="bf16", activation="none", residual=True, keep=False, turned=False, back=False),
        # The matrix cores' work: a wide layer with its residual over a fitting batch.
        _dense("dense-65536", 65_536, 4096, 4096, dtype="bf16", activation="gelu", residual=True, keep=False, turned=False, back=False),
        # Odd columns in 32 bits, the product kept for the way back.
        _dense("dense-odd-f32", 100_003, 50, 129, dtype="f32", activation="silu", residual=True, keep=True, turned=False, back=False),
        # All gradients of a shared layer over text embeddings.
        _dense("dense-back-65536", 65_536, 768, 2048, dtype="bf16", activation="silu", residual=False, keep=False, turned=False, back=True),
        # The norm over a map's many small tensors (launches and the host are most of it), and over large experts in 16 bits.
        {"name": "norm-120-tensors", "kind": "norm", "tensors": 120, "largest": 65_536, "dtype": "f32", "scaled": False},
        {"name": "norm-large", "kind": "norm", "tensors": 5, "largest": 200_000_003, "dtype": "bf16", "scaled": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "route", "dense", "dense", "dense", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "norm":
        tensors = _log(rng, 1, 200)
        return {"kind": kind, "tensors": tensors, "largest": min(200_000_003, _log(rng, 1, 200_000_003 * 2 // tensors)), "dtype": dtype, "scaled": rng.random() < 0.5}
    if kind == "route":
        groups = rng.choice([1, 1, 4, 8, rng.randint(2, 16)])
        each = rng.choice([8, 16, 32, _log(rng, 2, 128)]) if groups > 1 else rng.choice([8, 50, 64, 256, _log(rng, 2, 1_024)])
        top = 1 if groups == 1 else rng.randint(1, groups)
        n = min(_log(rng, 1, 500_000), 100_000_000 // (groups * each))
        return {"kind": kind, "n": n, "experts": groups * each, "k": rng.randint(1, min(8, top * each)), "groups": groups, "top_groups": top, "best": rng.choice([1, 2]),
                "score": rng.choice(["sigmoid", "sigmoid", "softmax"]), "bias": rng.random() < 0.8, "normalize": rng.random() < 0.7, "scale": rng.choice([1.0, 2.5]),
                "dtype": dtype, "gradient": rng.random() < 0.5}
    d, out = rng.choice([50, 128, 768, 4_096, _log(rng, 1, 8_192)]), rng.choice([2, 64, 256, 2_048, _log(rng, 1, 8_192)])
    back = rng.random() < 0.4
    # no more than a quarter of the largest listed product's operations, a sixteenth in 32 bits, where the matrix cores are slower
    most = (5e11 if dtype != "f32" else 5e10) / (2.0 if back else 1.0)
    n = max(1, min(_log(rng, 1, 262_144), int(most / (2.0 * d * out)), 500_000_000 // max(d, out)))
    return {"kind": kind, "n": n, "d": d, "out": out, "dtype": dtype, "activation": rng.choice(["none", "relu", "silu", "gelu"]), "residual": rng.random() < 0.5 and not back,
            "keep": rng.random() < 0.3 and not back, "turned": rng.random() < 0.3, "back": back}


def _sizes(case):
    """Numbers of elements of the tensors: the largest, and ever smaller ones with odd sizes among them."""
    return [max(1, int(case["largest"] / (1 + i) ** 1.3) - (i % 3)) for i in range(case["tensors"])]


# ---- inputs


def _randn(shape, scale, dtype, g):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"case": case}
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind == "norm":
        state["grads"] = [_randn(size, 1e-3, dtype, g) for size in _sizes(case)]
        state["scale"] = torch.full((1,), 1.0 / 1024.0, device="cuda") if case["scaled"] else None   # what a loss scaled by 1024 leaves to undo
        # half of what the norm is about: the step is clipped
        state["most"] = 0.5e-3 * math.sqrt(sum(_sizes(case))) * (1.0 / 1024.0 if case["scaled"] else 1.0)
        return state
    if kind == "route":
        n, experts, k = case["n"], case["experts"], case["k"]
        level = torch.randn(experts, generator=g, device="cuda").sub_(1.0)
        logits = torch.randn(n, experts, generator=g, device="cuda").mul_(1.5).add_(level)
        if n >= 64:
            logits[torch.randperm(n, generator=g, device="cuda")[:n // 64]] = -math.inf
        state["logits"] = logits.to(dtype)
        state["bias"] = _randn(experts, 0.02, torch.float32, g) if case["bias"] else None
        state["dweights"] = _randn((n, k), 1.0, torch.float32, g)
        return state
    n, d, out = case["n"], case["d"], case["out"]
    state["x"] = _randn((n, d), 1.0, dtype, g)
    w = _randn((d, out) if case["turned"] else (out, d), d ** -0.5, dtype, g)
    state["w"] = w.t() if case["turned"] else w                # weights kept either way round
    if case["back"]:
        state["z"], state["dy"] = _randn((n, out), 1.0, dtype, g), _randn((n, out), 1.0, dtype, g)
    else:
        state["bias"] = _randn(out, 0.1, dtype, g)
        state["residual"] = _randn((n, out), 1.0, dtype, g) if case["residual"] else None
    return state


# ---- the plain forms


def _largest(values, k, none):
    """Indices of the k largest of every row, the lowest index first among equals; `none` where only -inf is left."""
    number = torch.arange(values.shape[1], device=values.device)
    left, chosen = values, []
    for _ in range(k):
        best = left.amax(1, keepdim=True)
        at = torch.where(left == best, number, values.shape[1]).amin(1, keepdim=True)
        chosen.append(torch.where(best > -math.inf, at, none))
        left = left.scatter(1, at, -math.inf)
    return torch.cat(chosen, 1)


def _plain_route(state, case):
    """Scores in 64 bits: what decides is a difference of scores, however small."""
    logits, bias = state["logits"], state["bias"]
    n, experts = logits.shape
    k, groups = case["k"], case["groups"]
    x = logits.double()
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.amax(1, keepdim=True)
    if case["score"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-x))
    else:
        s = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
        s = s / s.sum(1, keepdim=True).clamp(min=1e-300)
    if bias is not None:
        c = torch.where(x > -math.inf, s + bias.double(), -math.inf)
        key = c
    else:
        c = torch.where(x > -math.inf, s, -math.inf)
        key = x
    if groups > 1:
        inside = (c if case["best"] == 2 or bias is not None else key).view(n, groups, experts // groups)
        if case["best"] == 1:
            total = inside.amax(2)
        else:
            first = inside.amax(2, keepdim=True)
            number = torch.arange(experts // groups, device=x.device)
            at = torch.where(inside == first, number, experts).amin(2, keepdim=True)
            second = inside.scatter(2, at, -math.inf).amax(2)
            total = first[:, :, 0] + torch.where(second > -math.inf, second, 0.0)
        open_ = torch.zeros(n, groups + 1, dtype=torch.bool, device=x.device).scatter_(1, _largest(total, case["top_groups"], groups), True)[:, :groups]
        key = torch.where(open_.repeat_interleave(experts // groups, 1), key, -math.inf)
    chosen = _largest(key, k, experts)
    there = chosen < experts
    at = torch.where(there, chosen, 0)
    picked = torch.where(there, s.gather(1, at), 0.0)
    weights = picked / picked.sum(1, keepdim=True).clamp(min=1e-300) if case["normalize"] else picked
    weights = (weights * case["scale"])
    flat = chosen.reshape(-1)
    by_expert, order = torch.sort(flat, stable=True)
    offsets = torch.searchsorted(by_expert, torch.arange(experts + 1, device=x.device))
    place = torch.empty_like(order).scatter_(0, order, torch.arange(n * k, device=x.device))
    out = {"experts": torch.where(there, chosen, -1).int(), "weights": weights.float(), "offsets": offsets.int(),
           "order": torch.where(by_expert < experts, order, -1).int(), "slots": torch.where(there.reshape(-1), place, -1).int().view(n, k)}
    if case["gradient"]:
        weights, s = weights.float(), s.float()
        dw = torch.where(there, state["dweights"], 0.0)
        inner = (weights * dw).sum(1, keepdim=True)
        if case["score"] == "softmax" and not case["normalize"]:
            given = torch.zeros_like(s).scatter_add_(1, at, dw)
            dl = s * (case["scale"] * given - inner)
        else:
            slope = torch.where(there, 1.0 - picked, 0.0).float() if case["score"] == "sigmoid" else 1.0
            each = slope * weights * (dw - inner / case["scale"] if case["normalize"] else dw)
            dl = torch.zeros_like(s).scatter_add_(1, at, torch.where(there, each, 0.0))
        out["dlogits"] = dl.to(logits.dtype)
        if bias is not None:
            count = offsets[1:] - offsets[:-1]
            out["bias"] = bias + BALANCE * torch.sign(offsets[-1] - experts * count).float()
    return out


def _act(z, name):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, name):
    if name == "relu":
        return (z > 0).float()
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _plain_dense(state, case):
    dtype, x, w = DTYPES[case["dtype"]], state["x"].float(), state["w"].float()
    if case["back"]:
        dz = state["dy"].float() * _slope(state["z"].float(), case["activation"])
        return {"dx": (dz @ w).to(dtype), "dw": (dz.t() @ x).to(dtype), "db": dz.sum(0)}
    z = x @ w.t() + state["bias"].float()
    y = _act(z, case["activation"])
    out = {"y": (y if state["residual"] is None else y + state["residual"].float()).to(dtype)}
    if case["keep"]:
        out["z"] = z.to(dtype)
    return out


def _plain_norm(state):
    """Squares in 64 bits: those of small gradients are lost in 32, and so are the last of a long sum."""
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in state["grads"]:
        d = g.double()
        total = total + (d * d).sum()
    scale = 1.0 if state["scale"] is None else state["scale"].double().reshape(())
    norm = torch.sqrt(total) * scale
    return {"norm": norm.float().reshape(1), "scale": (torch.where(norm <= state["most"], 1.0, state["most"] / norm) * scale).float().reshape(1)}


# ---- a pass


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["kind"] == "route":
        return _plain_route(state, case)
    return _plain_dense(state, case) if case["kind"] == "dense" else _plain_norm(state)


def _run_own(state, case):
    import paper_2505_15511_amd as nomad
    if case["kind"] == "norm":
        norm, scale = nomad.gradient_norm(state["grads"], max_norm=state["most"], grad_scale=state["scale"])
        return {"norm": norm, "scale": scale}
    if case["kind"] == "route":
        r = nomad.route_scored(state["logits"], case["k"], score=case["score"], bias=state["bias"], groups=case["groups"], top_groups=case["top_groups"],
                               group_best=case["best"], normalize=case["normalize"], scale=case["scale"])
        out = {"experts": r.experts, "weights": r.weights, "offsets": r.offsets, "order": r.order, "slots": r.slots}
        if case["gradient"]:
            out["dlogits"] = nomad.route_scored_gradient(state["logits"], r, state["dweights"], score=case["score"], normalize=case["normalize"], scale=case["scale"])
            if state["bias"] is not None:
                out["bias"] = nomad.balance_bias(state["bias"], r.offsets, BALANCE)
        return out
    if case["back"]:
        dx, dw, db = nomad.dense_gradient(state["dy"], state["x"], state["w"], activation=case["activation"], z=state["z"])
        return {"dx": dx, "dw": dw, "db": db}
    y = nomad.dense_product(state["x"], state["w"], bias=state["bias"], activation=case["activation"], residual=state["residual"], keep=case["keep"])
    return {"y": y[0], "z": y[1]} if case["keep"] else {"y": y}


# ---- what a pass cannot do without


def work(case):
    """Bytes: inputs once, outputs once; operations: 2 a multiply-add."""
    size = float({"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]])
    if case["kind"] == "norm":
        total = float(sum(_sizes(case)))
        return {"bytes": total * size + 8.0, "flops": 2.0 * total}
    if case["kind"] == "route":
        n, experts, k = float(case["n"]), float(case["experts"]), float(case["k"])
        back = (4.0 * n * k + n * experts * size) if case["gradient"] else 0.0
        return {"bytes": n * experts * size + 16.0 * n * k + 8.0 * experts + back, "flops": 4.0 * n * experts}
    n, d, out = float(case["n"]), float(case["d"]), float(case["out"])
    if case["back"]:
        read = n * d + out * d + n * out * (1.0 if case["activation"] == "none" else 2.0)
        return {"bytes": size * (read + n * d + out * d) + 4.0 * out, "flops": 4.0 * n * d * out}
    return {"bytes": size * (n * d + out * d + out + n * out * (1.0 + case["residual"] + case["keep"])), "flops": 2.0 * n * d * out}


# ---- 64 bits


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "norm":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in state["grads"]))
        scale = 1.0 if state["scale"] is None else float(state["scale"][0])
        norm *= scale
        out = {"norm": norm, "scale": scale * min(1.0, state["most"] / norm if norm > 0.0 else 1.0)}
        return {name: torch.tensor([value], dtype=torch.float64, device="cuda") for name, value in out.items()}
    if case["kind"] == "route":
        return _exact_route(state, case)
    x, w, name = state["x"].double(), state["w"].double(), case["activation"]
    if case["back"]:
        z, dz = state["z"].double(), state["dy"].double()
        if name == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif name == "silu":
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        elif name == "gelu":
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi))
        return {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t(), x), "db": torch.mv(dz.t(), torch.ones(case["n"], dtype=torch.float64, device="cuda"))}
    z = torch.addmm(state["bias"].double(), x, w.t())
    y = z.clamp(min=0) if name == "relu" else z * torch.sigmoid(z) if name == "silu" else z * torch.special.ndtr(z) if name == "gelu" else z
    out = {"y": y if state["residual"] is None else y + state["residual"].double()}
    if case["keep"]:
        out["z"] = z
    return out


def _exact_route(state, case):
    """From a stable order of every row's sums, the logarithms of the scores and their derivatives."""
    x = torch.nan_to_num(state["logits"].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    n, experts = x.shape
    k, groups, scale = case["k"], case["groups"], case["scale"]
    there = x > -math.inf
    log_s = torch.nn.functional.logsigmoid(x) if case["score"] == "sigmoid" else torch.nan_to_num(torch.log_softmax(x, 1), nan=-math.inf)
    by = x if state["bias"] is None else torch.where(there, torch.exp(log_s) + state["bias"].double(), -math.inf)
    if groups > 1:
        sums = by if state["bias"] is not None or case["best"] == 1 else torch.where(there, torch.exp(log_s), -math.inf)
        inside = torch.sort(sums.view(n, groups, -1), dim=2, descending=True).values[:, :, :case["best"]]
        total = inside[:, :, 0] + (torch.nan_to_num(inside[:, :, 1:], neginf=0.0).sum(2))
        rank = torch.argsort(torch.argsort(-total, dim=1, stable=True), dim=1)
        by = torch.where((rank < case["top_groups"])[:, :, None].expand(n, groups, experts // groups).reshape(n, experts), by, -math.inf)
    chosen = torch.argsort(-by, dim=1, stable=True)[:, :k]
    has = torch.gather(by, 1, chosen) > -math.inf
    picked = torch.where(has, torch.gather(log_s, 1, chosen), -math.inf)
    if case["normalize"]:
        share = torch.nan_to_num(torch.softmax(picked, 1), nan=0.0)
    else:
        share = torch.where(has, torch.exp(picked), 0.0)
    out = {"experts": None, "weights": scale * share, "offsets": None, "order": None, "slots": None}
    if case["gradient"]:
        dw = torch.where(has, state["dweights"].double(), 0.0) * scale
        back = share * (dw - (share * dw).sum(1, keepdim=True) if case["normalize"] else dw)   # of the logarithms of the chosen scores
        given = torch.zeros_like(x).scatter_add_(1, chosen, torch.where(has, back, 0.0))
        if case["score"] == "sigmoid":
            out["dlogits"] = given * torch.sigmoid(-x)
        else:
            out["dlogits"] = given - torch.where(there, torch.exp(log_s), 0.0) * given.sum(1, keepdim=True)
        if state["bias"] is not None:
            count = torch.bincount(chosen[has], minlength=experts)
            out["bias"] = state["bias"].double() + BALANCE * torch.sign(count.sum() - experts * count).double()
    return out
