"""The operators of a learned map as measurable cases: the router that sends a vector to the experts of a map's regions,
the experts' matrix products over ragged groups of rows with their gradients, the experts together as a map places or
is fitted, and the AdamW step over a map's tensors.

Inputs have the shapes that a partition gives: experts get rows in proportion to Dirichlet(1) weights, as clusters do,
and a row in 64 is padding, whose logits are all -inf."""
import math

import torch

own = False          # whether run() makes the framework's calls; its package is imported where they are made

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256          # elements that share a scale of the 8-bit states
LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 7


def _rows(kind, name, n, experts, k, **more):
    return {"name": name, "kind": kind, "n": n, "experts": experts, "k": k, **more}


def listed():
    return [
        # One vector asks for its region of a map of 256: the latency of a call.
        _rows("route", "route-1", 1, 256, 2, dtype="f32", gradient=False, normalize=True),
        # A million vectors over the default partition, one pass of fitting: the weights' gradient goes back to the logits.
        _rows("route", "route-1m", 1_000_000, 256, 2, dtype="f32", gradient=True, normalize=True),
        # A single vector through the first layer of its two experts: reads two experts' weights.
        _rows("product", "product-1", 1, 64, 2, d=768, out=2048, dtype="bf16", activation="silu"),
        # A batch of queries, about every expert asked and few rows each.
        _rows("product", "product-48", 48, 64, 2, d=768, out=2048, dtype="f16", activation="silu"),
        # The first layer over a quarter of a million text embeddings: the matrix cores' work.
        _rows("product", "product-262144", 262_144, 64, 2, d=768, out=2048, dtype="bf16", activation="silu"),
        # Odd columns in 32 bits: 50 columns, one expert a region of a small map.
        _rows("product", "product-odd-f32", 100_003, 50, 2, d=50, out=129, dtype="f32", activation="relu"),
        # Gradients of rows, weights and bias in fitting, 256 ragged experts.
        _rows("gradients", "gradients-100k", 100_003, 256, 2, d=768, out=512, dtype="bf16"),
        # Gradients at odd sizes in 32 bits.
        _rows("gradients", "gradients-odd-f32", 20_011, 50, 2, d=129, out=50, dtype="f32"),
        # New vectors placed on a map: router, both layers, the weighted sum.
        _rows("place", "place-100", 100, 50, 2, d=50, hidden=128, out=2, dtype="f32", fit=False),
        # A step of fitting the map of 128 columns, with every gradient.
        _rows("place", "fit-65536", 65_536, 256, 2, d=128, hidden=256, out=2, dtype="f32", fit=True),
        # The step over many small tensors (a map's layers, heads and biases): launches are most of it.
        {"name": "adamw-120-tensors", "kind": "adamw", "tensors": 120, "largest": 65_536, "dtype": "f32", "bits": 32},
        # The step over large experts in 16 bits with states in 8.
        {"name": "adamw-8bit", "kind": "adamw", "tensors": 5, "largest": 50_331_648, "dtype": "bf16", "bits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "product", "product", "gradients", "gradients", "place", "adamw"])
    if kind == "adamw":
        tensors = _log(rng, 1, 200)
        return {"kind": kind, "tensors": tensors, "largest": min(50_331_648, _log(rng, 100, 50_331_648 * 4 // tensors)), "dtype": rng.choice(["f32", "bf16", "f16"]),
                "bits": rng.choice([32, 8])}
    experts = rng.choice([8, 10, 50, 64, 256, _log(rng, 2, 1_024)])
    k = rng.randint(1, min(4, experts))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "route":
        n = min(_log(rng, 1, 1_000_000), 256_000_000 // experts)
        return {"kind": kind, "n": n, "experts": experts, "k": k, "dtype": dtype, "gradient": rng.random() < 0.5, "normalize": rng.random() < 0.7}
    d = rng.choice([50, 64, 128, 768, _log(rng, 2, 1_024)])
    out = rng.choice([2, 64, 256, 512, 2_048, _log(rng, 2, 2_048)])
    # no more than a quarter of the largest listed product's operations in 32 bits, where the matrix cores are slower
    most = 8e11 if dtype != "f32" else 5e10
    n = max(1, min(_log(rng, 1, 262_144), int(most / (2.0 * k * d * out))))
    if kind == "product":
        return {"kind": kind, "n": n, "experts": experts, "k": k, "d": d, "out": out, "dtype": dtype, "activation": rng.choice(["none", "relu", "silu", "gelu"])}
    if kind == "gradients":
        return {"kind": kind, "n": n, "experts": experts, "k": k, "d": d, "out": out, "dtype": dtype}
    hidden = _log(rng, 16, 512)
    n = max(1, min(n, int(2e10 / (6.0 * k * d * hidden))))
    return {"kind": kind, "n": n, "experts": experts, "k": k, "d": min(d, 256), "hidden": hidden, "out": rng.choice([2, 3]), "dtype": "f32", "fit": rng.random() < 0.5}


def _sizes(case):
    """Numbers of elements of the tensors of a step: the largest, and ever smaller ones with odd sizes among them."""
    return [max(1, int(case["largest"] / (1 + i) ** 1.3) - (i % 3)) for i in range(case["tensors"])]


# ---- inputs


def _logits(case, g):
    """Gumbel noise on the logarithms of Dirichlet(1) weights: the best expert of a row is a draw from those weights."""
    n, experts = case["n"], case["experts"]
    share = -torch.log(torch.rand(experts, generator=g, device="cuda").clamp_(min=1e-30))
    logits = -torch.log(-torch.log(torch.rand(n, experts, generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)))
    logits += torch.log(share / share.sum())
    if n >= 64:
        logits[torch.randperm(n, generator=g, device="cuda")[:n // 64]] = -math.inf
    return logits


def _randn(shape, scale, dtype, g):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"case": case}
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind == "adamw":
        for name in ("params", "grads", "first", "second"):
            state[name] = []
        for size in _sizes(case):
            state["params"].append(_randn(size, 0.05, dtype, g))
            grad = _randn(size, 1e-3, dtype, g)
            state["grads"].append(grad)
            # averages as some steps leave them: sizes of gradients differ from row to row
            spread = torch.exp(torch.randn(-(-size // 64), generator=g, device="cuda")).repeat_interleave(64)[:size]
            m = 3e-4 * spread * torch.randn(size, generator=g, device="cuda")
            v = (1e-3 * spread) ** 2 * (0.5 + torch.rand(size, generator=g, device="cuda"))
            state["first"].append(_encode_first(m) if case["bits"] == 8 else m)
            state["second"].append(_encode_second(v) if case["bits"] == 8 else v)
        return state
    logits = _logits(case, g)
    n, experts, k = case["n"], case["experts"], case["k"]
    if kind in ("route", "place"):
        state["logits"] = logits.to(dtype)
    if kind == "route":
        state["dweights"] = _randn((n, k), 1.0, torch.float32, g)
        return state
    if kind == "place":
        d, h, out = case["d"], case["hidden"], case["out"]
        state["x"] = _randn((n, d), 1.0, dtype, g)
        state["w1"], state["b1"] = _randn((experts, h, d), d ** -0.5, dtype, g), _randn((experts, h), 0.1, dtype, g)
        state["w2"], state["b2"] = _randn((experts, out, h), h ** -0.5, dtype, g), _randn((experts, out), 0.1, dtype, g)
        state["dy"] = _randn((n, out), 1.0, dtype, g)
        return state
    # products: the grouping is there already (a layer in the middle of a map), and the host knows the groups' ends
    _, _, state["offsets"], state["order"], _ = _plain_route(logits, k, True)
    state["ends"] = state["offsets"].tolist()
    d, out = case["d"], case["out"]
    state["x"] = _randn((n, d), 1.0, dtype, g)
    state["w"] = _randn((experts, out, d), d ** -0.5, dtype, g)
    if kind == "product":
        state["bias"] = _randn((experts, out), 0.1, dtype, g)
    else:
        state["dy"] = _randn((n * k, out), 1.0, dtype, g)
    return state


# ---- the plain forms


def _plain_route(logits, k, normalize):
    """Experts, weights, group offsets, order (slots by expert, -1 behind them) and slots' places (-1: no expert)."""
    n, experts = logits.shape
    left = logits.float()
    left = torch.where(left.isnan(), -math.inf, left)
    number = torch.arange(experts, device=left.device)
    top = left.amax(1, keepdim=True)
    total = torch.exp(left - top).sum(1, keepdim=True)
    values, chosen = [], []
    for _ in range(k):                                        # the best that is left, the lowest index among equals
        best = left.amax(1, keepdim=True)
        at = torch.where(left == best, number, experts).amin(1, keepdim=True)
        left = left.scatter(1, at, -math.inf)
        values.append(best)
        chosen.append(at)
    values, chosen = torch.cat(values, 1), torch.cat(chosen, 1)
    there = values > -math.inf
    e = torch.exp(values - top)
    weights = torch.where(there, e / (torch.where(there, e, 0.0).sum(1, keepdim=True) if normalize else total), 0.0)
    chosen = torch.where(there, chosen, experts).reshape(-1)
    by_expert, order = torch.sort(chosen, stable=True)
    offsets = torch.searchsorted(by_expert, torch.arange(experts + 1, device=left.device))
    place = torch.empty_like(order).scatter_(0, order, torch.arange(n * k, device=left.device))
    slots = torch.where(there.reshape(-1), place, -1)
    order = torch.where(by_expert < experts, order, -1)
    experts_of = torch.where(there.reshape(-1), chosen, -1)
    return experts_of.int().view(n, k), weights, offsets.int(), order.int(), slots.int().view(n, k)


def _plain_route_gradient(logits, experts_of, weights, dweights, normalize):
    there = experts_of >= 0
    dw = torch.where(there, dweights, 0.0)
    inner = (weights * dw).sum(1, keepdim=True)
    at = torch.where(there, experts_of, 0).long()
    if normalize:
        g = torch.zeros(logits.shape, device=logits.device)
        return g.scatter_add_(1, at, torch.where(there, weights * (dw - inner), 0.0)).to(logits.dtype)
    x = logits.float()
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    p = e / e.sum(1, keepdim=True).clamp(min=1e-30)
    return (p * (torch.zeros_like(p).scatter_add_(1, at, dw) - inner)).to(logits.dtype)


def _act(z, name):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _gathered(x, order, k):
    """The rows of x in the order of the groups, float32; zeros behind them."""
    return torch.where((order >= 0)[:, None], x.float()[torch.div(order.clamp(min=0), k, rounding_mode="floor").long()], 0.0)


def _plain_product(rows, w, ends, bias=None, activation="none"):
    """Groups differ in length: a matrix product each, into its rows of the result."""
    y = torch.zeros(rows.shape[0], w.shape[1], device=rows.device)
    w = w.float()
    for e in range(w.shape[0]):
        if ends[e] < ends[e + 1]:
            z = rows[ends[e]:ends[e + 1]] @ w[e].t()
            y[ends[e]:ends[e + 1]] = z if bias is None else z + bias[e].float()
    if activation != "none":
        y[:ends[-1]] = _act(y[:ends[-1]], activation)
    return y


def _plain_weight_gradient(dy, rows, ends):
    dw = torch.zeros(len(ends) - 1, dy.shape[1], rows.shape[1], device=dy.device)
    db = torch.zeros(len(ends) - 1, dy.shape[1], device=dy.device)
    for e in range(len(ends) - 1):
        if ends[e] < ends[e + 1]:
            part = dy[ends[e]:ends[e + 1]]
            torch.mm(part.t(), rows[ends[e]:ends[e + 1]], out=dw[e])
            db[e] = part.sum(0)
    return dw, db


def _plain_place(state):
    case, dtype, k = state["case"], DTYPES[state["case"]["dtype"]], state["case"]["k"]
    experts_of, weights, offsets, order, slots = _plain_route(state["logits"], k, True)
    ends = offsets.tolist()                                   # (products of whole groups need their sizes on the host)
    rows = _gathered(state["x"], order, k)
    z = _plain_product(rows, state["w1"], ends, state["b1"])
    h = z / (1.0 + torch.exp(-z))
    h[ends[-1]:] = 0.0
    o = _plain_product(h, state["w2"], ends, state["b2"])
    there = (slots >= 0)[:, :, None]
    at = slots.clamp(min=0).long()
    picked = torch.where(there, o[at], 0.0)
    y = (weights[:, :, None] * picked).sum(1)
    if not case["fit"]:
        return {"y": y.to(dtype)}
    dy = state["dy"].float()
    dweights = (dy[:, None, :] * picked).sum(2)
    slot = order.clamp(min=0).long()
    do = torch.where((order >= 0)[:, None], weights.reshape(-1)[slot][:, None] * dy[torch.div(slot, k, rounding_mode="floor")], 0.0)
    dw2, db2 = _plain_weight_gradient(do, h, ends)
    s = 1.0 / (1.0 + torch.exp(-z))
    dz = _plain_product(do, state["w2"].transpose(1, 2), ends) * (s * (1.0 + z * (1.0 - s)))
    dw1, db1 = _plain_weight_gradient(dz, rows, ends)
    dx = torch.where(there, _plain_product(dz, state["w1"].transpose(1, 2), ends)[at], 0.0).sum(1)
    dlogits = _plain_route_gradient(state["logits"], experts_of, weights, dweights, True)
    return {"y": y.to(dtype), "dx": dx.to(dtype), "dlogits": dlogits, "dw1": dw1.to(dtype), "db1": db1, "dw2": dw2.to(dtype), "db2": db2}


# The 8-bit states: blocks of 256 elements with the largest magnitude s as their scale (0 where it is no normal number);
# first averages as s (c/127) |c/127| with c in -127..127, second averages as s (c/255)^4 with c in 0..255, 0 only for 0.
# A code is the whole number whose borders c - 1/2 and c + 1/2, squared (to the fourth), hold the scaled value between them.

SMALLEST = 2.0 ** -126


def _blocks(x):
    n = x.numel()
    padded = torch.zeros(-(-n // BLOCK) * BLOCK, device=x.device)
    padded[:n] = x
    return padded.view(-1, BLOCK)


def _scaled(magnitude, most):
    """(scale of every block, magnitudes with the scale at `most`)."""
    s = magnitude.amax(1)
    s = torch.where(s < SMALLEST, 0.0, s)
    factor = torch.where(s > 0, torch.full_like(s, most) / torch.where(s > 0, s, 1.0), 0.0)
    return s, magnitude * factor[:, None]


def _encode_first(m):
    b = _blocks(m)
    s, t = _scaled(b.abs(), 127.0 ** 2)
    c = torch.round(torch.sqrt(t))
    up, down = c + 0.5, c - 0.5
    c = c + (t >= up * up).float() - (t < down * down).float() * (c > 0)
    return (torch.sign(b) * c).view(-1)[:m.numel()].to(torch.int8), s


def _encode_second(v):
    b = _blocks(v)
    s, t = _scaled(b, 255.0 ** 4)
    c = torch.round(torch.sqrt(torch.sqrt(t)))
    up, down = c + 0.5, c - 0.5
    up, down = up * up, down * down
    c = c + (t >= up * up).float() - (t < down * down).float() * (c > 0)
    c = torch.where((b > 0) & (s > 0)[:, None], c.clamp(min=1.0), 0.0)
    return c.view(-1)[:v.numel()].to(torch.uint8), s


def _decode_first(codes, s):
    t = codes.float() * (1.0 / 127.0)
    return (t * t.abs()) * s.repeat_interleave(BLOCK)[:codes.numel()]


def _decode_second(codes, s):
    t = codes.float() * (1.0 / 255.0)
    t = t * t
    return (t * t) * s.repeat_interleave(BLOCK)[:codes.numel()]


def _f32(x):
    """x as the nearest float32 (scalars of a step are rounded once)."""
    return float(torch.tensor(x, dtype=torch.float32))


def _plain_adamw(state):
    """Every operation rounds once in 32 bits, in this order, so that codes of 8 bits are the same numbers wherever it runs."""
    bits8 = state["case"]["bits"] == 8
    keep, rate = _f32(1.0 - LR * DECAY), _f32(LR / (1.0 - BETA1 ** STEP))
    root = _f32(1.0 / math.sqrt(1.0 - BETA2 ** STEP))
    for i, (p, grad) in enumerate(zip(state["params"], state["grads"])):
        m, v = state["first"][i], state["second"][i]
        g = grad.float()
        m_new = (_decode_first(*m) if bits8 else m) * _f32(BETA1) + g * _f32(1.0 - BETA1)
        v_new = (_decode_second(*v) if bits8 else v) * _f32(BETA2) + (g * g) * _f32(1.0 - BETA2)
        step = (m_new * rate) / (torch.sqrt(v_new) * root + _f32(EPS))
        p.copy_(p.float() * keep - step)
        if bits8:
            for old, new in ((m, _encode_first(m_new)), (v, _encode_second(v_new))):
                old[0].copy_(new[0])
                old[1].copy_(new[1])
        else:
            m.copy_(m_new)
            v.copy_(v_new)
    if bits8:
        return {"params": _some(state["params"]), "first": _some([_decode_first(*m) for m in state["first"]]), "second": _some([_decode_second(*v) for v in state["second"]])}
    return {"params": _some(state["params"]), "first": _some(state["first"]), "second": _some(state["second"])}


def _some(tensors):
    """All tensors where they are few; where they are many, twelve that include the largest and the smallest."""
    return list(tensors) if len(tensors) <= 12 else [tensors[i * (len(tensors) - 1) // 11] for i in range(12)]


# ---- a pass


def run(state):
    case = state["case"]
    kind, k = case["kind"], case.get("k")
    if own:
        return _run_own(state, case, kind, k)
    if kind == "adamw":
        return _plain_adamw(state)
    if kind == "route":
        got = _plain_route(state["logits"], k, case["normalize"])
        out = dict(zip(("experts", "weights", "offsets", "order", "slots"), got))
        if case["gradient"]:
            out["dlogits"] = _plain_route_gradient(state["logits"], got[0], got[1], state["dweights"], case["normalize"])
        return out
    if kind == "place":
        return _plain_place(state)
    dtype = DTYPES[case["dtype"]]
    rows = _gathered(state["x"], state["order"], k)
    if kind == "product":
        return _plain_product(rows, state["w"], state["ends"], state["bias"], case["activation"]).to(dtype)
    dy = state["dy"].float()
    dx = _plain_product(dy, state["w"].transpose(1, 2), state["ends"])
    dw, db = _plain_weight_gradient(dy, rows, state["ends"])
    return {"dx": dx.to(dtype), "dw": dw.to(dtype), "db": db}


def _run_own(state, case, kind, k):
    import paper_2505_15511_amd as nomad
    if kind == "adamw":
        nomad.adamw_step(state["params"], state["grads"], state["first"], state["second"], step=STEP, lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY)
        first, second = _some(state["first"]), _some(state["second"])
        if case["bits"] == 8:
            first, second = nomad.adamw_state_values(first), nomad.adamw_state_values(second)
        return {"params": _some(state["params"]), "first": first, "second": second}
    if kind == "route":
        r = nomad.route(state["logits"], k, normalize=case["normalize"])
        out = {"experts": r.experts, "weights": r.weights, "offsets": r.offsets, "order": r.order, "slots": r.slots}
        if case["gradient"]:
            out["dlogits"] = nomad.route_gradient(state["logits"], r, state["dweights"], normalize=case["normalize"])
        return out
    if kind == "product":
        return nomad.grouped_product(state["x"], state["w"], state["offsets"], bias=state["bias"], activation=case["activation"], order=state["order"], per_row=k)
    if kind == "gradients":
        dx = nomad.grouped_product(state["dy"], state["w"].transpose(1, 2), state["offsets"])
        dw, db = nomad.grouped_weight_gradient(state["dy"], state["x"], state["offsets"], order=state["order"], per_row=k)
        return {"dx": dx, "dw": dw, "db": db}
    from paper_2505_15511_amd import placement
    r = nomad.route(state["logits"], k)
    layers = (state["w1"], state["b1"], state["w2"], state["b2"])
    if not case["fit"]:
        return {"y": placement.experts(state["x"], r, *layers)}
    y, kept = placement.experts(state["x"], r, *layers, keep=True)
    g = placement.experts_gradient(state["dy"], state["x"], r, *layers, kept)
    dlogits = nomad.route_gradient(state["logits"], r, g["dweights"])
    return {"y": y, "dx": g["dx"], "dlogits": dlogits, "dw1": g["dw1"], "db1": g["db1"], "dw2": g["dw2"], "db2": g["db2"]}


# ---- what a pass cannot do without


def work(case):
    """Bytes: inputs once (of the experts' weights no more than rows can ask for), outputs once; operations: 2 a multiply-add."""
    size = float({"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]])
    if case["kind"] == "adamw":
        sizes = _sizes(case)
        total = float(sum(sizes))
        state = 8.0 if case["bits"] == 32 else 2.0 + 8.0 / BLOCK
        shown = sum(_some(sizes)) * (2.0 + 8.0) if case["bits"] == 8 else 0.0
        return {"bytes": total * (3 * size + 2 * state) + shown, "flops": 14.0 * total}
    n, experts, k = float(case["n"]), float(case["experts"]), float(case["k"])
    rows = n * k
    asked = min(experts, rows)
    logits = n * experts * size
    routing = 16.0 * rows + 4.0 * experts
    if case["kind"] == "route":
        back = (4.0 * rows + logits) if case["gradient"] else 0.0
        return {"bytes": logits + routing + back, "flops": 2.0 * n * experts}
    d, out = float(case["d"]), float(case["out"])
    if case["kind"] == "product":
        return {"bytes": size * (n * d + asked * out * (d + 1) + rows * out) + 4.0 * rows, "flops": 2.0 * rows * d * out}
    if case["kind"] == "gradients":
        return {"bytes": size * (rows * out + n * d + asked * out * d + rows * d + experts * out * d) + 4.0 * (rows + experts * out), "flops": 4.0 * rows * d * out}
    layers = case["hidden"] * (d + out + 1.0) + out
    back = 2.0 if case["fit"] else 0.0
    more = (n * (out + d) * size + logits + experts * layers * size) if case["fit"] else 0.0
    return {"bytes": logits + size * (n * d + asked * layers + n * out) + more, "flops": 2.0 * rows * case["hidden"] * (d + out) * (1.0 + back)}


# ---- 64 bits


def _groups(logits, k):
    """(expert of every slot or -1) from the definition: a stable order of every row's logits."""
    x = torch.nan_to_num(logits.double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    best = torch.argsort(-x, dim=1, stable=True)[:, :k]
    value = torch.gather(x, 1, best)
    return torch.where(value == -math.inf, -1, best), x


def exact(case, seed):
    state = prepare(case, seed)
    kind, k = case["kind"], case.get("k")
    if kind == "adamw":
        params, firsts, seconds = [], [], []
        for i in _some(list(range(len(state["params"])))):
            p, g = state["params"][i].double(), state["grads"][i].double()
            m, v = state["first"][i], state["second"][i]
            if case["bits"] == 8:
                t, u = m[0].double() / 127.0, v[0].double() / 255.0
                m = t * t.abs() * m[1].double().repeat_interleave(BLOCK)[:p.numel()]
                v = u ** 4 * v[1].double().repeat_interleave(BLOCK)[:p.numel()]
            m = BETA1 * m.double() + (1.0 - BETA1) * g
            v = BETA2 * v.double() + (1.0 - BETA2) * g * g
            hat = (m / (1.0 - BETA1 ** STEP)) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + EPS)
            params.append(p - LR * (hat + DECAY * p))
            firsts.append(None if case["bits"] == 8 else m)   # (codes are a matter of the rounding before them)
            seconds.append(None if case["bits"] == 8 else v)
        return {"params": params, "first": firsts, "second": seconds}
    if kind in ("route", "place"):
        chosen, x = _groups(state["logits"], k)
        e = torch.exp(x - x.amax(1, keepdim=True).clamp(min=-1e300))
        picked = torch.where(chosen >= 0, torch.gather(e, 1, chosen.clamp(min=0)), 0.0)
        total = picked.sum(1, keepdim=True) if case.get("normalize", True) else e.sum(1, keepdim=True)
        weights = picked / total.clamp(min=1e-300)
    if kind == "route":
        out = {"experts": None, "weights": weights, "offsets": None, "order": None, "slots": None}
        if case["gradient"]:
            dw = torch.where(chosen >= 0, state["dweights"].double(), 0.0)
            given = torch.zeros_like(x).scatter_add_(1, chosen.clamp(min=0), dw)
            inner = (weights * dw).sum(1, keepdim=True)
            full = e / total.clamp(min=1e-300)
            if case["normalize"]:
                full = full * torch.zeros_like(x).scatter_add_(1, chosen.clamp(min=0), (chosen >= 0).double())
            out["dlogits"] = full * (given - inner)
        return out
    if kind == "place":
        return _exact_place(state, case, chosen, weights)
    ends, order = state["ends"], state["order"].long()
    x = state["x"].double()
    source = torch.div(order[:ends[-1]], k, rounding_mode="floor")
    total = case["n"] * k
    if kind == "product":
        if 2.0 * total * case["d"] * case["out"] > 1e13:
            return None
        y = torch.zeros(total, case["out"], dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            a, b = ends[e], ends[e + 1]
            z = torch.addmm(state["bias"][e].double(), x[source[a:b]], state["w"][e].double().t())
            name = case["activation"]
            y[a:b] = z.clamp(min=0) if name == "relu" else z * torch.sigmoid(z) if name == "silu" else z * torch.special.ndtr(z) if name == "gelu" else z
        return y
    dx = torch.zeros(total, case["d"], dtype=torch.float64, device="cuda")
    dw = torch.zeros(case["experts"], case["out"], case["d"], dtype=torch.float64, device="cuda")
    db = torch.zeros(case["experts"], case["out"], dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        a, b = ends[e], ends[e + 1]
        dy = state["dy"][a:b].double()
        dx[a:b] = dy @ state["w"][e].double()
        dw[e] = dy.t() @ x[source[a:b]]
        db[e] = dy.sum(0)
    return {"dx": dx, "dw": dw, "db": db}


def _exact_place(state, case, chosen, weights):
    """Expert by expert over the slots that chose it, gradients by the chain rule written out."""
    x, dy = state["x"].double(), state["dy"].double()
    names = ("w1", "b1", "w2", "b2")
    y, dx = torch.zeros(x.shape[0], case["out"], dtype=torch.float64, device="cuda"), torch.zeros_like(x)
    dweights = torch.zeros_like(weights)
    grads = {"d" + name: torch.zeros_like(state[name], dtype=torch.float64) for name in names}
    for e in range(case["experts"]):
        w1, b1, w2, b2 = (state[name][e].double() for name in names)
        i, j = torch.nonzero(chosen == e, as_tuple=True)
        z = x[i] @ w1.t() + b1
        gate = torch.sigmoid(z)
        h = z * gate
        o = h @ w2.t() + b2
        w = weights[i, j][:, None]
        y.index_add_(0, i, w * o)
        dweights[i, j] = (dy[i] * o).sum(1)
        do = w * dy[i]
        dz = (do @ w2) * (gate + h * (1.0 - gate))
        grads["dw2"][e], grads["db2"][e] = do.t() @ h, do.sum(0)
        grads["dw1"][e], grads["db1"][e] = dz.t() @ x[i], dz.sum(0)
        dx.index_add_(0, i, dz @ w1)
    if not case["fit"]:
        return {"y": y}
    inner = (weights * dweights).sum(1, keepdim=True)
    dlogits = torch.zeros(state["logits"].shape, dtype=torch.float64, device="cuda")
    dlogits.scatter_add_(1, chosen.clamp(min=0), torch.where(chosen >= 0, weights * (dweights - inner), 0.0))
    return {"y": y, "dx": dx, "dlogits": dlogits, **grads}
