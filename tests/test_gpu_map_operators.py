"""The learned map's operators against the float64 oracle, at the sizes, layouts and masks where they can go wrong.

Tolerances are bounds: a float32 sum of K terms in any order is off by at most (K + 8) 2^-24 times the sum of their absolute
values; an activation passes that on with a slope of at most 1.13 and adds its own rounding, a few units of 2^-24 times
(1 + |z|) |z|; the result is rounded once to its type."""
import math

import numpy as np
import pytest
import torch

import paper_2505_15511_amd as nomad
from oracle import map_oracle as mo
from paper_2505_15511_amd import NomadError

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def note(msg):
    print(msg, flush=True)


def host(t):
    return t.detach().to("cpu", torch.float64).numpy()


def near(got, want, bound, dtype, what):
    got = host(got)
    smallest = 2.0 ** -25 if dtype == F16 else 1e-37
    limit = bound + UNIT[dtype] * (np.abs(want) + bound) + smallest
    worst = np.max(np.abs(got - want) / limit) if got.size else 0.0
    note(f"  {what}: {worst:.3f} of the bound")
    assert got.shape == want.shape and worst <= 1.0


def lengths(kind, groups, total, rng):
    """Rows of every group."""
    if kind == "even":
        return [total // groups] * groups
    if kind == "empty":
        return [0] * groups
    if kind == "one":
        return [total if e == groups // 2 else 0 for e in range(groups)]
    cut = np.sort(rng.integers(0, total + 1, size=groups - 1))        # ragged, empty groups among them
    return np.diff(np.concatenate([[0], cut, [total]])).tolist()


def grouping(kind, groups, total, rng, spare=0):
    offsets = np.concatenate([[0], np.cumsum(lengths(kind, groups, total, rng))]).astype(np.int32)
    return offsets, int(offsets[-1]) + spare


def randn(shape, dtype, rng, scale=1.0):
    return torch.from_numpy(rng.normal(size=shape) * scale).to("cuda", dtype)


# ---- routing

ROUTES = [(1, 256, 2, F32), (1, 3, 3, F32), (7, 10, 2, BF16), (64, 50, 4, F16), (300, 64, 1, F32), (1025, 256, 2, BF16), (3000, 50, 8, F32), (700, 1000, 3, F16),
          (5000, 8, 2, F32), (260, 1029, 5, F32), (40, 16384, 2, BF16), (2, 1, 1, F32), (33000, 33, 2, F32)]


def check_routing(logits, k, normalize):
    r = nomad.route(logits, k, normalize=normalize)
    experts, weights, offsets, order, slots = mo.route(host(logits), k, normalize)
    for name, got, want in (("experts", r.experts, experts), ("offsets", r.offsets, offsets), ("order", r.order, order), ("slots", r.slots, slots)):
        assert np.array_equal(got.cpu().numpy(), want), name
    # exponentials are good to 2 units each and their sum to one per term
    terms = k if normalize else logits.shape[1]
    assert np.array_equal(np.isnan(host(r.weights)), np.isnan(weights))
    near(torch.nan_to_num(r.weights), np.nan_to_num(weights), (terms + 8) * U32 * np.nan_to_num(weights), F32, "weights")
    return r, weights


@pytest.mark.parametrize("n,experts,k,dtype", ROUTES)
@pytest.mark.parametrize("normalize", [True, False])
def test_routing(n, experts, k, dtype, normalize):
    note(f"route n={n} E={experts} k={k} {dtype} {normalize}")
    rng = np.random.default_rng(n + experts)
    x = rng.normal(size=(n, experts)).astype(np.float32)
    x[rng.random((n, experts)) < 0.2] = -np.inf                       # masked experts
    x[rng.random((n, experts)) < 0.05] = np.nan
    x[rng.random((n, experts)) < 0.2] = 0.5                           # ties
    x[rng.random((n, experts)) < 0.05] = -0.0
    x[rng.random((n, experts)) < 0.05] = 0.0
    x[rng.random(n) < 0.1] = -np.inf                                  # rows without any
    logits = torch.from_numpy(x).to("cuda", dtype)
    r, weights = check_routing(logits, k, normalize)
    dw = torch.from_numpy(rng.normal(size=(n, k)).astype(np.float32)).cuda()
    got = nomad.route_gradient(logits, r, dw, normalize=normalize)
    want = mo.route_gradient(host(logits), r.experts.cpu().numpy(), weights, host(dw), normalize)
    size = np.abs(host(dw)).max() * (experts + 24) * U32
    near(got, want, size, dtype, "dlogits")


@pytest.mark.parametrize("n,experts,k,dtype", [(1, 16384, 8, F32), (2, 16384, 8, BF16), (1, 16377, 8, F16), (1, 16376, 8, F32), (2, 16370, 7, F32)])
def test_routing_of_a_row_or_two_over_many_experts(n, experts, k, dtype):
    """On either side of what one workgroup has LDS for."""
    note(f"route n={n} E={experts} k={k} {dtype}")
    rng = np.random.default_rng(n + experts + k)
    for normalize in (True, False):
        check_routing(torch.from_numpy(rng.normal(size=(n, experts)).astype(np.float32)).to("cuda", dtype), k, normalize)


def test_routing_strides_extremes_and_rows_that_all_want_one_expert():
    note("route strides")
    rng = np.random.default_rng(1)
    base = torch.from_numpy(rng.normal(size=(900, 70)).astype(np.float32)).cuda()
    check_routing(base[:, 3:67], 2, True)                              # rows apart, not aligned
    check_routing(base[::3, :64], 2, True)
    check_routing(base[5:6].expand(600, 70), 2, False)                 # one row for all: every row the same experts
    lowest = torch.finfo(F32).min
    x = torch.full((400, 12), lowest, device="cuda")                   # a mask of the lowest number is a number: chosen in order
    x[:, 5] = 1.0
    check_routing(x, 3, True)
    x[7, 2] = float("inf")
    check_routing(x, 3, True)
    r = nomad.route(torch.empty(0, 9, device="cuda"), 2)
    assert r.offsets.tolist() == [0] * 10 and r.order.numel() == 0


def test_routing_many_rows_against_torch():
    note("route 400000 x 128")
    logits = torch.randn(400_000, 128, device="cuda")
    logits[::97] = -float("inf")
    r = nomad.route(logits, 2)
    top = torch.sort(logits, dim=1, descending=True, stable=True)
    want = torch.where(top.values[:, :2] > -float("inf"), top.indices[:, :2], -1).int()
    assert torch.equal(r.experts, want)
    flat = torch.where(want >= 0, want, 128).reshape(-1)
    by, order = torch.sort(flat, stable=True)
    assert torch.equal(r.order, torch.where(by < 128, order, -1).int())
    assert torch.equal(r.offsets.long(), torch.searchsorted(by, torch.arange(129, device="cuda")))
    assert torch.equal(r.slots.reshape(-1)[r.order[:int(r.offsets[-1])].long()], torch.arange(int(r.offsets[-1]), device="cuda").int())


# ---- products

#: (groups, rows, in, out, type, how rows fall into groups)
PRODUCTS = [(1, 1, 1, 1, F32, "ragged"), (3, 1, 50, 129, F32, "one"), (4, 300, 50, 129, F32, "ragged"), (2, 130, 7, 3, BF16, "ragged"), (5, 700, 64, 2, BF16, "ragged"),
            (8, 1000, 128, 256, BF16, "ragged"), (8, 5, 768, 96, F16, "ragged"), (3, 600, 129, 130, F16, "ragged"), (1, 513, 768, 72, BF16, "even"), (70, 900, 64, 40, F32, "ragged"),
            (5, 33_000, 72, 520, BF16, "ragged"), (130, 9_000, 264, 272, F16, "ragged"), (2, 20_000, 256, 136, BF16, "ragged"), (3, 9_000, 20, 12, F32, "one"),
            (6, 400, 2, 260, F32, "ragged"), (4, 0, 16, 16, BF16, "empty"), (3, 64, 24, 24, BF16, "empty"), (2, 2100, 200, 264, BF16, "ragged"), (1030, 2000, 40, 24, F16, "ragged"),
            (9000, 5000, 40, 24, F16, "ragged")]


@pytest.mark.parametrize("groups,total,inner,out,dtype,kind", PRODUCTS)
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("gathered", [False, True])
def test_product(groups, total, inner, out, dtype, kind, turned, gathered):
    note(f"product groups={groups} rows={total} {inner}->{out} {dtype} {kind} turned={turned} gathered={gathered}")
    rng = np.random.default_rng(groups + total + inner)
    spare = 0 if total == 0 else 37
    offsets, places = grouping(kind, groups, total, rng, spare)
    per_row = 3
    x_rows = max(1, places // 2) if gathered else places
    x = randn((x_rows, inner), dtype, rng)
    order = None
    if gathered:
        order = rng.integers(-1, x_rows * per_row + 4, size=places).astype(np.int32)      # (some rows that there are not)
    w = randn((groups, inner, out) if turned else (groups, out, inner), dtype, rng, inner ** -0.5)
    w = w.transpose(1, 2) if turned else w
    bias = randn((groups, out), dtype, rng)
    go, gd = torch.from_numpy(offsets).cuda(), None if order is None else torch.from_numpy(order).cuda()
    for activation in ("none", "relu", "silu", "gelu"):
        y, z = nomad.grouped_product(x, w, go, bias, activation, order=gd, per_row=per_row, keep=True)
        want_y, want_z, size = mo.product(host(x), host(w), offsets, host(bias), activation, order, per_row, places=places)
        bound = (inner + 8) * U32 * size
        near(z, want_z, bound, dtype, "z")
        near(y, want_y, 1.13 * bound + 8 * U32 * (1 + np.abs(want_z)) * np.abs(want_z), dtype, activation)
        if activation != "none":
            dz = nomad.grouped_product(x, w, go, activation=activation, order=gd, per_row=per_row, slope_at=z)
            zz = host(z)
            want, plain, size = mo.product(host(x), host(w), offsets, None, activation, order, per_row, slope_at=zz, places=places)
            near(dz, want, 1.13 * (inner + 8) * U32 * size + 16 * U32 * (1 + np.abs(zz)) * np.abs(plain), dtype, "slope of " + activation)
    assert (y[int(offsets[-1]):] == 0).all() and (z[int(offsets[-1]):] == 0).all()
    wide = nomad.grouped_product(x, w, go, order=gd, per_row=per_row, out_dtype=F32)
    want, _, size = mo.product(host(x), host(w), offsets, None, None, order, per_row, places=places)
    near(wide, want, (inner + 8) * U32 * size, F32, "float32 results")


@pytest.mark.parametrize("groups,total,inner,out,dtype,kind", PRODUCTS)
@pytest.mark.parametrize("gathered", [False, True])
def test_weight_gradient(groups, total, inner, out, dtype, kind, gathered):
    note(f"gradient groups={groups} rows={total} {inner}->{out} {dtype} {kind} gathered={gathered}")
    rng = np.random.default_rng(groups + total + inner + 1)
    offsets, places = grouping(kind, groups, total, rng, 0 if total == 0 else 37)
    per_row = 2
    x_rows = max(1, places // 2) if gathered else places
    x, dy = randn((x_rows, inner), dtype, rng), randn((places, out), dtype, rng)
    order = rng.integers(-1, x_rows * per_row + 3, size=places).astype(np.int32) if gathered else None
    dy[int(offsets[-1]):] = float("nan")                               # rows of no group are not looked at
    go, gd = torch.from_numpy(offsets).cuda(), None if order is None else torch.from_numpy(order).cuda()
    want, want_b, size, size_b = mo.weight_gradient(np.nan_to_num(host(dy)), host(x), offsets, order, per_row)
    longest = max(1, int(np.diff(offsets).max()))
    for out_dtype in {dtype, F32}:
        dw, db = nomad.grouped_weight_gradient(dy, x, go, order=gd, per_row=per_row, out_dtype=out_dtype)
        near(dw, want, (longest + 8) * U32 * size, out_dtype, "dw")
        near(db, want_b, (longest + 8) * U32 * size_b, F32, "db")
    again, none = nomad.grouped_weight_gradient(dy, x, go, order=gd, per_row=per_row, bias=False, out_dtype=F32)
    assert none is None and torch.equal(again, nomad.grouped_weight_gradient(dy, x, go, order=gd, per_row=per_row, out_dtype=F32)[0])


@pytest.mark.parametrize("rows", [6, 700])
@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_activations_of_float32_results(rows, name, dtype):
    """Relative to the result, by unit matrices, which leave z exact.  The exponential, a sum and a quotient take a few roundings; GELU's argument
    is rounded before erfc, whose relative slope is z^2; a slope's two terms add up with their errors."""
    note(f"float32 {name} rows={rows} {dtype}")
    z = torch.cat([torch.linspace(-9, 9, rows * 64 - 64, dtype=torch.float64), torch.logspace(-30, 0, 32, dtype=torch.float64), -torch.logspace(-30, 0, 32, dtype=torch.float64)])
    x = z.reshape(rows, 64).cuda().to(dtype)
    z, eye, offsets = host(x), torch.eye(64, device="cuda", dtype=dtype)[None], torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    limit = 16 * U32 * (1.0 if name == "silu" else 1.0 + 0.25 * z * z)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        want, first, second = z * s, s, z * s * (1.0 - s)
    else:
        erfc, density = np.vectorize(math.erfc), np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
        first, second = 0.5 * erfc(-z / math.sqrt(2.0)), z * density
        want = z * first
    got = host(nomad.grouped_product(x, eye, offsets, activation=name, out_dtype=F32))
    off = np.abs(got - want) / np.maximum(np.abs(want), 1e-37)
    note(f"  {np.max(off / limit):.3f} of the bound")
    assert np.all(off <= limit)
    ones = torch.ones(1, 64, 1, device="cuda", dtype=dtype)
    got = host(nomad.grouped_product(torch.ones(rows, 1, device="cuda", dtype=dtype), ones, offsets, activation=name, slope_at=x, out_dtype=F32))
    off = np.abs(got - (first + second)) / (np.abs(first) + np.abs(second))
    note(f"  slope: {np.max(off / limit):.3f} of the bound")
    assert np.all(off <= limit)


@pytest.mark.parametrize("rows", [6, 700])
@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_activations_of_16_bit_results(rows, name, dtype):
    """The result's rounding hides all but a 16th of it: 2^-16 of the result beside that, which the smallest numbers keep too."""
    note(f"16 bits {name} rows={rows} {dtype}")
    x = torch.linspace(-9, 9, rows * 64, dtype=torch.float64).reshape(rows, 64).cuda().to(dtype)
    z, eye, offsets = host(x), torch.eye(64, device="cuda", dtype=dtype)[None], torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    want = z / (1.0 + np.exp(-z)) if name == "silu" else 0.5 * z * np.vectorize(math.erfc)(-z / math.sqrt(2.0))
    off = np.abs(host(nomad.grouped_product(x, eye, offsets, activation=name)) - want)
    limit = (UNIT[dtype] + 2.0 ** -16) * np.abs(want) + (2.0 ** -25 if dtype == F16 else 1e-37)
    note(f"  {np.max(off / limit):.3f} of the bound")
    assert np.all(off <= limit)


def test_product_layouts():
    """Rows apart, columns off by an element, weights shared by all groups, and numbers that are not finite in rows of others."""
    note("product layouts")
    rng = np.random.default_rng(9)
    for dtype in (F32, BF16, F16):
        offsets = np.array([0, 100, 100, 260], np.int32)
        go = torch.from_numpy(offsets).cuda()
        big, wide = randn((300, 150), dtype, rng), randn((3, 90, 151), dtype, rng, 0.1)
        for x, w in ((big[:260, 8:136], wide[:, :64, 8:136]), (big[:260, 1:130], wide[:, 3:70, 1:130]), (big[:260, :64], wide[:1, :80, :64].expand(3, 80, 64)),
                     (big[0:1, :64].expand(260, 64), wide[:, ::2, :64]), (big[:260, :72], wide[:, :80, ::2][:, :, :72].contiguous().transpose(1, 2)[:, :72].transpose(1, 2))):
            want, _, size = mo.product(host(x), host(w), offsets)
            near(nomad.grouped_product(x, w, go), want, (x.shape[1] + 8) * U32 * size, dtype, f"strides {x.stride()} {w.stride()}")
        x, w = randn((260, 40), dtype, rng), randn((3, 33, 40), dtype, rng)
        clean = nomad.grouped_product(x, w, go)
        x[7], w[1] = float("nan"), float("inf")                        # one row, and the weights of the group without rows
        x[250, 3] = float("inf")
        got = nomad.grouped_product(x, w, go)
        keep = torch.ones(260, dtype=torch.bool, device="cuda")
        keep[[7, 250]] = False
        assert torch.equal(got[keep], clean[keep]) and got[7].isnan().all() and not got[250].isfinite().any()


def test_product_rows_and_weights_beyond_32_bits():
    """Rows and weights more than 2^32 bytes from their base, and a stride that alone passes 2^31 elements."""
    note("product far rows")
    rng = np.random.default_rng(10)
    n, d = 1_200_000, 2_048                                            # 4.9e9 bytes of bfloat16
    x = torch.zeros(n, d, dtype=BF16, device="cuda")
    x[-300:] = randn((300, d), BF16, rng)
    w = torch.zeros(3, 16, d, dtype=BF16, device="cuda")
    w[2] = randn((16, d), BF16, rng, d ** -0.5)
    offsets = np.array([0, 0, n - 300, n], np.int32)
    y = nomad.grouped_product(x, w, torch.from_numpy(offsets).cuda())
    want, _, size = mo.product(host(x[-300:]), host(w[2:]), [0, 300])
    near(y[-300:], want, (d + 8) * U32 * size, BF16, "far rows")
    assert (y[:-300] == 0).all()
    dw, db = nomad.grouped_weight_gradient(y, x, torch.from_numpy(offsets).cuda())
    want, want_b, size, size_b = mo.weight_gradient(host(y[-300:]), host(x[-300:]), [0, 300])
    near(dw[2:], want, 308 * U32 * size, BF16, "dw of far rows")
    assert (dw[:2] == 0).all()
    del x
    apart = torch.zeros(2 ** 31 + 4096, dtype=BF16, device="cuda")
    far = apart.as_strided((2, 64), (2 ** 31 + 64, 1))
    far.copy_(randn((2, 64), BF16, rng))
    near(nomad.grouped_product(far, w[2:, :, :64], torch.tensor([0, 2], dtype=torch.int32, device="cuda")),
         mo.product(host(far), host(w[2:, :, :64]), [0, 2])[0], 72 * U32 * mo.product(host(far), host(w[2:, :, :64]), [0, 2])[2], BF16, "rows far apart")


def test_offsets_that_are_not_groups_stay_in_range():
    note("odd offsets")
    rng = np.random.default_rng(11)
    x, w = randn((50, 32), BF16, rng), randn((3, 32, 32), BF16, rng)
    for odd in ([0, 60, 2 ** 31 - 1, 70], [0, -5, 20, 50], [0, 30, 10, 50]):
        y = nomad.grouped_product(x, w, torch.tensor(odd, dtype=torch.int32, device="cuda"))
        dw, _ = nomad.grouped_weight_gradient(y, x, torch.tensor(odd, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert y.shape == (50, 32) and dw.shape == (3, 32, 32)


# ---- the weighted sum


@pytest.mark.parametrize("n,k,d,dtype", [(1, 1, 1, F32), (300, 2, 2, F32), (130, 3, 50, BF16), (77, 8, 768, F16), (1000, 2, 129, F32), (65, 4, 1028, BF16)])
def test_combine(n, k, d, dtype):
    note(f"combine n={n} k={k} d={d} {dtype}")
    rng = np.random.default_rng(n + d)
    x = rng.normal(size=(n, 9)).astype(np.float32)
    x[rng.random((n, 9)) < 0.5] = -np.inf
    r = nomad.route(torch.from_numpy(x).cuda(), k)
    values, dy = randn((n * k, d), dtype, rng), randn((n, d), dtype, rng)
    slots, weights = r.slots.cpu().numpy(), host(r.weights)
    for w in (r.weights, None):
        want = mo.combine(host(values), slots, weights if w is not None else None)
        size = mo.combine(np.abs(host(values)), slots, weights if w is not None else None)
        near(nomad.combine(values, r.slots, w), want, (k + 2) * U32 * size, dtype, "y")
        dv, dw = nomad.combine_gradient(dy, values, r.slots, w, order=r.order)
        want_v, want_w = mo.combine_gradient(host(dy), host(values), slots, weights if w is not None else None)
        near(dv, want_v, 2 * U32 * np.abs(want_v), dtype, "dvalues")
        near(dw, want_w, (d + 8) * U32 * mo.combine_gradient(np.abs(host(dy)), np.abs(host(values)), slots)[1], F32, "dweights")
    only, none = nomad.combine_gradient(dy, values, r.slots, r.weights, order=r.order, need_dweights=False)
    assert none is None and torch.equal(only, nomad.combine_gradient(dy, values, r.slots, r.weights, order=r.order)[0])
    wide = torch.cat([values, values], 1)[:, 1:1 + d] if d > 1 else values
    near(nomad.combine(wide, r.slots), mo.combine(host(wide), slots), (k + 2) * U32 * mo.combine(np.abs(host(wide)), slots), dtype, "rows apart")


# ---- AdamW

PAIRS = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]


def sizes_and_views(dtype, g_dtype, rng):
    """Tensors of odd sizes, none among them, one that begins off every border, more than a launch's arguments hold."""
    sizes = [1, 7, 256, 257, 2048, 0, 5000, 2049, 4096] + [3 + i for i in range(70)]
    params, grads = [], []
    for i, n in enumerate(sizes):
        p, g = randn((n + 1,), dtype, rng), randn((n + 1,), g_dtype, rng, 0.01)
        params.append(p[1:] if i % 2 else p[:n])
        grads.append(g[1:] if i % 3 == 1 else g[:n])
    return params, grads


@pytest.mark.parametrize("dtype,g_dtype", PAIRS)
@pytest.mark.parametrize("scaled", [False, True])
def test_adamw_in_32_bits(dtype, g_dtype, scaled):
    note(f"adamw 32 {dtype} {g_dtype} scaled={scaled}")
    rng = np.random.default_rng(21)
    params, grads = sizes_and_views(dtype, g_dtype, rng)
    states = [nomad.adamw_state(p) for p in params]
    scale = torch.tensor([0.25], device="cuda") if scaled else None
    want = [(host(p), host(m), host(v)) for p, (m, v) in zip(params, states)]
    for step in (1, 2, 3):
        nomad.adamw_step(params, grads, [s[0] for s in states], [s[1] for s in states], step, lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1, grad_scale=scale)
        for i, (p, g, (m, v)) in enumerate(zip(params, grads, states)):
            before = want[i]
            wp, wm, wv = mo.adamw(*(before[0], host(g)), before[1], before[2], step, 0.01, 0.9, 0.99, 1e-6, 0.1, 0.25 if scaled else 1.0)
            # each step's roundings: a few of float32, and one of the parameter's type (from where the GPU's own values were)
            assert np.abs(host(m) - wm).max(initial=0) <= 8 * U32 * np.abs(wm).max(initial=0) + 1e-30
            assert np.abs(host(v) - wv).max(initial=0) <= 8 * U32 * np.abs(wv).max(initial=0) + 1e-30
            assert np.all(np.abs(host(p) - wp) <= UNIT[dtype] * np.abs(wp) + 2.0 ** -25 * (dtype == F16) + 16 * U32 * (np.abs(before[0]) + 0.2))
            want[i] = (host(p), host(m), host(v))


@pytest.mark.parametrize("dtype,g_dtype", PAIRS)
def test_adamw_in_8_bits(dtype, g_dtype):
    """Codes are the nearest of their kind: each stands for a value within half a step of the average it rounds, at every step
    from the values that the codes before it stood for."""
    note(f"adamw 8 {dtype} {g_dtype}")
    rng = np.random.default_rng(22)
    params, grads = sizes_and_views(dtype, g_dtype, rng)
    states = [nomad.adamw_state(p, 8) for p in params]
    for step in (1, 2, 3):
        before = [(host(p), mo.decode_first(*(t.cpu().numpy() for t in m)), mo.decode_second(*(t.cpu().numpy() for t in v))) for p, (m, v) in zip(params, states)]
        nomad.adamw_step(params, grads, [s[0] for s in states], [s[1] for s in states], step, lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
        shown = nomad.adamw_state_values([s[0] for s in states]), nomad.adamw_state_values([s[1] for s in states])
        for i, (p, g, (m, v)) in enumerate(zip(params, grads, states)):
            wp, wm, wv = mo.adamw(before[i][0], host(g), before[i][1], before[i][2], step, 0.01, 0.9, 0.99, 1e-6, 0.1)
            assert np.all(np.abs(host(p) - wp) <= UNIT[dtype] * np.abs(wp) + 2.0 ** -25 * (dtype == F16) + 32 * U32 * (np.abs(before[i][0]) + 0.2))
            if not wm.size:
                continue
            for got, want, codes, most, power, decode in ((shown[0][i], wm, m, 127, 2, mo.decode_first), (shown[1][i], wv, v, 255, 4, mo.decode_second)):
                c, s = codes.codes.cpu().numpy().astype(np.float64), codes.scales.cpu().numpy().astype(np.float64)
                assert np.abs(host(got) - decode(codes.codes.cpu().numpy(), codes.scales.cpu().numpy())).max() <= 8 * U32 * np.abs(host(got)).max()
                top = np.array([np.abs(want[b:b + 256]).max() for b in range(0, want.size, 256)])
                assert np.all(np.abs(s - top) <= 8 * U32 * top)
                t = np.abs(want) * (most ** power / np.repeat(s, 256)[:want.size])
                a = np.abs(c)
                slack = 64 * U32 * t                                   # the average's own rounding
                low = np.maximum(a - 0.5, 0.0) ** power * (1.0 if power == 2 else (a > 1))
                assert np.all(t + slack >= low) and np.all(t - slack <= (a + 0.5) ** power) and np.all((c != 0) | (want == 0) | (power == 2))
                assert np.all((np.sign(c) == np.sign(want)) | (c == 0))


def test_adamw_8_bits_zeros_and_values_that_are_not_finite():
    note("adamw 8 special values")
    p, g = torch.ones(1024, device="cuda"), torch.zeros(1024, device="cuda")
    m, v = nomad.adamw_state(p, 8)
    nomad.adamw_step([p], [g], [m], [v], 1, lr=0.1, weight_decay=0.0)
    assert (p == 1).all() and (m.scales == 0).all() and (v.codes == 0).all()
    g[300], g[600] = float("nan"), float("inf")
    nomad.adamw_step([p], [g], [m], [v], 2, lr=0.1, weight_decay=0.0)
    first = nomad.adamw_state_values([m])[0]
    assert first[256:512].isnan().all() and first[512:768].isnan().all() and (first[:256] == 0).all() and (first[768:] == 0).all()
    assert p[300].isnan() and (p[:256] == 1).all()
    tiny = torch.full((256,), 1e-30, device="cuda")                    # squares below the smallest normal number
    q = torch.ones(256, device="cuda")
    m, v = nomad.adamw_state(q, 8)
    nomad.adamw_step([q], [tiny], [m], [v], 1, lr=0.1, eps=1e-8, weight_decay=0.0)
    assert (v.scales == 0).all() and (m.codes == 127).all() and torch.isfinite(q).all()


#: scales of a block around and below the ones whose quotients 127^2 / s and 255^4 / s are no float32 numbers (4.7e-35, 1.24e-29)
SMALL_SCALES = [1.2e-38, 1e-37, 1e-36, 4e-35, 5e-35, 1e-33, 1e-30, 1.2e-29, 1.3e-29, 8e-28, 9e-28, 1e-20]


@pytest.mark.parametrize("which", ["first", "second"])
def test_adamw_8_bits_small_scales(which):
    """One block a scale, its averages four decades and both signs: codes are those of the borders at every scale.  An average is the
    sum and product of a few float32 numbers: good to some 2^-24 of itself and some 2^-149, its distance to a border likewise."""
    note(f"adamw 8 small scales of the {which} averages")
    rng = np.random.default_rng(23)
    beta1, beta2 = 0.5, 0.75                                           # (powers of two: the products add no rounding of their own)
    g = np.concatenate([(s / 0.5 if which == "first" else np.sqrt(s / 0.25)) * np.where(np.arange(256) == 0, 1.0, 10.0 ** rng.uniform(-4, 0, 256)) * rng.choice([-1.0, 1.0], 256)
                        for s in SMALL_SCALES]).astype(np.float32)
    p, grad = torch.ones(g.size, device="cuda"), torch.from_numpy(g).cuda()
    m, v = nomad.adamw_state(p, 8)
    nomad.adamw_step([p], [grad], [m], [v], 1, lr=0.1, betas=(beta1, beta2), weight_decay=0.0)
    g = g.astype(np.float64)
    state, average, encode, most, power = (m, 0.5 * g, mo.encode_first, 127, 2) if which == "first" else (v, 0.25 * g * g, mo.encode_second, 255, 4)
    codes, scales = state.codes.cpu().numpy().astype(np.float64), state.scales.cpu().numpy().astype(np.float64)
    want, want_scales, t = encode(average)
    assert np.all(np.abs(scales - want_scales) <= 8 * U32 * want_scales + 2.0 ** -147)
    slack = 64 * U32 * t + 2.0 ** -147 * most ** power / np.repeat(want_scales, 256)
    a = np.abs(codes)
    assert np.all(t - slack < (a + 0.5) ** power)
    assert np.all((t + slack >= np.maximum(a - 0.5, 0.0) ** power) | ((power == 4) & (a == 1)))
    assert np.all((np.sign(codes) == np.sign(average)) | (codes == 0))
    assert np.mean(codes == want) > 0.95 and np.array_equal(codes.reshape(-1, 256)[:, 0], want.reshape(-1, 256)[:, 0])
    # and they decode to the average, within half a code's step
    shown = host(nomad.adamw_state_values([state])[0])
    step = np.repeat(want_scales, 256) * ((a + 0.5) ** power - np.maximum(a - 0.5, 0.0) ** power) / most ** power
    assert np.all(np.abs(shown - average) <= step * 1.001 + 2.0 ** -147)


def test_adamw_8_bits_averages_that_are_not_finite():
    """A block with an average that is NaN or infinite is NaN, of the first averages and of the second; its neighbours are not."""
    note("adamw 8 averages that are not finite")
    g = torch.full((1280,), 0.5, device="cuda")
    g[300], g[600], g[900] = float("nan"), float("inf"), 1e25          # (the square of the last one passes float32)
    p = torch.ones(1280, device="cuda")
    m, v = nomad.adamw_state(p, 8)
    nomad.adamw_step([p], [g], [m], [v], 1, lr=0.1, weight_decay=0.0)
    first, second = nomad.adamw_state_values([m])[0].view(5, 256), nomad.adamw_state_values([v])[0].view(5, 256)
    assert first[1:3].isnan().all() and first[[0, 3, 4]].isfinite().all()
    assert second[1:4].isnan().all() and second[[0, 4]].isfinite().all()


@pytest.mark.parametrize("eps", [1e-8, 1e-30, 0.0])
@pytest.mark.parametrize("bits,dtype", [(32, F32), (8, F32), (32, BF16), (8, BF16)])
def test_adamw_steps_of_small_gradients(eps, bits, dtype):
    """The step from the averages that the state shows, down to the smallest v that is not zero: from zero a parameter becomes minus
    its step, which takes half a dozen roundings, the hardware's reciprocal and root among them."""
    note(f"adamw small gradients eps={eps} bits={bits} {dtype}")
    g = torch.logspace(-20.5, 2, 4096, device="cuda", dtype=torch.float64).float()
    g[1::2] *= -1.0
    p = torch.zeros(4096, device="cuda", dtype=dtype)
    m, v = nomad.adamw_state(p, bits)
    nomad.adamw_step([p], [g], [m], [v], 1, lr=0.25, betas=(0.5, 0.75), eps=eps, weight_decay=0.0)
    first = 0.5 * host(g)                                              # exact: a power of two
    d2 = (host(g).astype(np.float32) * host(g).astype(np.float32)).astype(np.float32)
    second = (d2 * np.float32(0.25)).astype(np.float64)                # as float32 holds it, denormal numbers too
    assert (second > 0).all() and (bits == 8 or np.array_equal(host(v), second))
    want = -0.25 * (first / 0.5) / (np.sqrt(second / 0.25) + eps)
    assert np.all(np.abs(host(p) - want) <= (16 * U32 + UNIT[dtype]) * np.abs(want))


@pytest.mark.parametrize("dtype,g_dtype", [(F32, F32), (BF16, BF16), (F16, F32)])
def test_adamw_dithered_codes(dtype, g_dtype):
    """Every code lies between the two borders that its element's draw gives, to the rounding of the average and of the borders."""
    note(f"adamw dithered {dtype} {g_dtype}")
    rng = np.random.default_rng(24)
    params, grads = sizes_and_views(dtype, g_dtype, rng)
    states = [nomad.adamw_state(p, 8) for p in params]
    for step in (1, 2, 2 ** 33 + 5):
        before = [(host(p), mo.decode_first(*(t.cpu().numpy() for t in m)), mo.decode_second(*(t.cpu().numpy() for t in v))) for p, (m, v) in zip(params, states)]
        nomad.adamw_step(params, grads, [s[0] for s in states], [s[1] for s in states], step, lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1, dither=True)
        for i, (p, g, (m, v)) in enumerate(zip(params, grads, states)):
            wp, wm, wv = mo.adamw(before[i][0], host(g), before[i][1], before[i][2], step, 0.01, 0.9, 0.99, 1e-6, 0.1)
            assert np.all(np.abs(host(p) - wp) <= UNIT[dtype] * np.abs(wp) + 2.0 ** -25 * (dtype == F16) + 32 * U32 * (np.abs(before[i][0]) + 0.2))
            if not wm.size:
                continue
            for want, codes, most, power, second in ((wm, m, 127, 2, False), (wv, v, 255, 4, True)):
                c, s = np.abs(codes.codes.cpu().numpy().astype(np.float64)), codes.scales.cpu().numpy().astype(np.float64)
                top = np.array([np.abs(want[b:b + 256]).max() for b in range(0, want.size, 256)])
                assert np.all(np.abs(s - top) <= 8 * U32 * top)
                t, u = np.abs(want) * (most ** power / np.repeat(s, 256)[:want.size]), mo.draws(want.size, step, second)

                def border(low):
                    return low ** power + u * ((low + 1.0) ** power - low ** power)
                slack = 64 * U32 * t
                assert np.all((t - slack <= border(c)) | (c == most)) and c.max() <= most
                assert np.all((t + slack >= border(c - 1.0)) | (c == 0) | (second & (c == 1)))
                sign = np.sign(codes.codes.cpu().numpy().astype(np.float64))
                assert np.all((sign == np.sign(want)) | (c == 0)) and np.all((c > 0) | (want == 0) | (not second))


def test_adamw_dithered_averages_follow_changing_gradients():
    """As in the oracle's test of the same name, by the kernel, with a third of the gradients ending altogether: their first averages reach
    0 (at code 1 a draw keeps it nine times in ten), where nearest codes stop at 9."""
    note("adamw dithered, 4,000 steps")
    n, steps, beta2 = 6144, 4000, 0.999
    kind = torch.arange(n, device="cuda") % 3
    p = torch.zeros(n, device="cuda")
    m, v = nomad.adamw_state(p, 8)
    early, late = torch.ones(n, device="cuda"), torch.where(kind == 0, 1.0, torch.where(kind == 1, 0.03, 0.0)).float()
    exact, variance = np.zeros(3), 0.0
    for step in range(1, steps + 1):
        nomad.adamw_step([p], [early if step <= 800 else late], [m], [v], step, lr=1e-3, betas=(0.9, beta2), weight_decay=0.0, dither=True)
        exact = beta2 * exact + (1 - beta2) * (np.ones(3) if step <= 800 else np.array([1.0, 0.03 ** 2, 0.0]))
        c = 255.0 * (exact[2] / exact[0]) ** 0.25
        variance += (1 - beta2) * (4 / c + 6 / c ** 2)
    shown, codes = host(nomad.adamw_state_values([v])[0]), m.codes.cpu().numpy()
    kind = kind.cpu().numpy()
    for which in (1, 2):
        of = shown[kind == which]
        note(f"  kind {which}: {of.mean() / exact[which] - 1:+.4f} of {6 * np.sqrt(variance / of.size):.4f}")
        assert abs(of.mean() / exact[which] - 1) < 6 * np.sqrt(variance / of.size)
    assert (codes[kind == 2] == 0).all() and (codes[kind == 0] == 127).all()


def test_adamw_dither_is_the_same_every_time_and_not_for_32_bits():
    note("adamw dither repeats")
    rng = np.random.default_rng(25)
    g = randn((5001,), F32, rng)
    got = []
    for step, stream in ((7, None), (7, torch.cuda.Stream().cuda_stream), (8, None)):
        p = torch.zeros(5001, device="cuda")
        m, v = nomad.adamw_state(p, 8)
        nomad.adamw_step([torch.zeros(3, device="cuda"), p], [g[:3].clone(), g], [nomad.adamw_state(g[:3], 8)[0], m], [nomad.adamw_state(g[:3], 8)[1], v], step, dither=True, stream=stream)
        torch.cuda.synchronize()
        got.append(torch.cat([m.codes.int(), v.codes.int()]))
    assert torch.equal(got[0], got[1]) and (got[0] != got[2]).float().mean() > 0.1
    with pytest.raises(ValueError):
        nomad.adamw_step([g], [g.clone()], [torch.zeros_like(g)], [torch.zeros_like(g)], 1, dither=True)


# ---- streams and refusals


def test_another_stream_and_a_graph():
    note("streams")
    rng = np.random.default_rng(30)
    logits, x = randn((500, 40), F32, rng), randn((500, 64), BF16, rng)
    w = randn((40, 48, 64), BF16, rng, 0.1)

    def whole(stream=None):
        r = nomad.route(logits, 2, stream=stream)
        y, z = nomad.grouped_product(x, w, r.offsets, activation="silu", order=r.order, per_row=2, keep=True, stream=stream)
        dw, db = nomad.grouped_weight_gradient(y, x, r.offsets, order=r.order, per_row=2, stream=stream)
        return nomad.combine(y, r.slots, r.weights, stream=stream), dw, db, z
    want = whole()
    side = torch.cuda.Stream()
    got = whole(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    whole()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = whole()
    for seed in (1, 2, 3):                                             # new inputs at every replay
        logits.copy_(torch.randn(500, 40, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        fresh = whole()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, fresh))


def test_another_stream_waits_for_the_current_one_and_the_host_does_not():
    note("another stream behind work of the current one")
    rng = np.random.default_rng(31)
    logits, big, product = randn((300, 40), F32, rng), torch.ones(8192, 8192, device="cuda"), torch.empty(8192, 8192, device="cuda")
    side = torch.cuda.Stream()
    want = nomad.route(logits, 2)
    nomad.route(logits, 2, stream=side.cuda_stream)
    torch.mm(big, big, out=product)
    torch.cuda.synchronize()
    fresh, done = torch.empty_like(logits), torch.cuda.Event()
    for _ in range(40):                                                # some 7 ms each
        torch.mm(big, big, out=product)
    fresh.copy_(logits)                                                # the input comes after all that
    done.record()
    got = nomad.route(fresh, 2, stream=side.cuda_stream)
    assert not done.query()                                            # the call is back, and the current stream still at work
    side.synchronize()
    assert done.query() and all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):                                      # the other way round: the default stream is the other one
        fresh = logits.clone()
        got = nomad.route(fresh, 2, stream=0)
        torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_graph_with_another_stream_in_it():
    note("a graph with another stream")
    rng = np.random.default_rng(32)
    logits, x, w = randn((500, 40), F32, rng), randn((500, 64), BF16, rng), randn((40, 48, 64), BF16, rng, 0.1)
    side = torch.cuda.Stream()

    def whole(stream):
        r = nomad.route(logits, 2)
        y = nomad.grouped_product(x, w, r.offsets, order=r.order, per_row=2, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(side)
        return nomad.combine(y, r.slots, r.weights)
    whole(side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = whole(side.cuda_stream)
    for seed in (1, 2, 3):
        logits.copy_(torch.randn(500, 40, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        fresh = whole(None)
        torch.cuda.synchronize()
        assert torch.equal(held, fresh)


def test_refusals():
    x, w = torch.zeros(10, 8, device="cuda"), torch.zeros(2, 4, 8, device="cuda")
    offsets = torch.tensor([0, 5, 10], dtype=torch.int32, device="cuda")
    logits = torch.zeros(10, 4, device="cuda")
    r = nomad.route(logits, 2)
    bad = [lambda: nomad.route(logits, 0), lambda: nomad.route(logits, 5), lambda: nomad.route(logits.double(), 2), lambda: nomad.route(logits.t(), 2),
           lambda: nomad.route(logits.cpu(), 2), lambda: nomad.route(torch.zeros(2, 16385, device="cuda"), 2), lambda: nomad.route(torch.zeros(2, 20, device="cuda"), 9),
           lambda: nomad.route_gradient(logits, r, torch.zeros(10, 3, device="cuda")), lambda: nomad.grouped_product(x, w[:, :, :7], offsets),
           lambda: nomad.grouped_product(x, w.half(), offsets), lambda: nomad.grouped_product(x, w, offsets[:2]), lambda: nomad.grouped_product(x, w, offsets.long()),
           lambda: nomad.grouped_product(x, w, offsets, activation="tanh"), lambda: nomad.grouped_product(x.t(), w, offsets),
           lambda: nomad.grouped_product(x, torch.zeros(2, 8, 16, device="cuda")[:, ::2, ::2], offsets), lambda: nomad.grouped_product(x, w, offsets, bias=torch.zeros(4, device="cuda")),
           lambda: nomad.grouped_product(x, w, offsets, out_dtype=F16), lambda: nomad.grouped_product(x, w, offsets, slope_at=torch.zeros(10, 4, device="cuda"), keep=True),
           lambda: nomad.grouped_product(x, w, offsets, order=torch.zeros(4, device="cuda")), lambda: nomad.grouped_product(x, w, offsets.cpu()),
           lambda: nomad.grouped_product(x, w, offsets, order=torch.zeros(4, dtype=torch.int32, device="cuda"), per_row=0),
           lambda: nomad.grouped_weight_gradient(torch.zeros(9, 4, device="cuda"), x, offsets), lambda: nomad.grouped_weight_gradient(torch.zeros(10, 4, device="cuda").half(), x, offsets),
           lambda: nomad.combine(x, torch.zeros(5, 2, device="cuda")), lambda: nomad.combine(x, r.slots, torch.zeros(10, 3, device="cuda")),
           lambda: nomad.combine_gradient(x, x, r.slots, order=r.order), lambda: nomad.adamw_state(x, 16),
           lambda: nomad.adamw_step([x], [x], [x], [], 1), lambda: nomad.adamw_step([x], [x.double()], [x], [x], 1), lambda: nomad.adamw_step([x], [x], [x.half()], [x], 1),
           lambda: nomad.adamw_step([x.t()], [x], [x], [x], 1), lambda: nomad.adamw_step([x], [x], [x.clone()], [nomad.adamw_state(x, 8)[1]], 1)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            note(f"refusal {i} did not happen")
    for f in (lambda: nomad.adamw_step([x], [x], [x.clone()], [x.clone()], 0), lambda: nomad.adamw_step([x], [x], [x.clone()], [x.clone()], 1, betas=(1.0, 0.9)),
              lambda: nomad.adamw_step([x], [x], [x.clone()], [x.clone()], 1, lr=float("nan"))):
        with pytest.raises(NomadError):
            f()
    nomad.adamw_step([], [], [], [], 1)


def test_refusals_of_other_shapes():
    """Tensors of another number of dimensions and the like are refused as the rest is, not by an IndexError on the way."""
    note("refusals of shapes")
    x, w = torch.zeros(10, 8, device="cuda"), torch.zeros(2, 4, 8, device="cuda")
    offsets, order = torch.tensor([0, 5, 10], dtype=torch.int32, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    r = nomad.route(torch.zeros(10, 4, device="cuda"), 2)
    none, line = torch.zeros((), device="cuda"), torch.zeros(10, device="cuda")
    bad = [lambda: nomad.route(line, 2), lambda: nomad.route(none, 1), lambda: nomad.route_gradient(x[:, :4], r._replace(experts=r.experts.view(-1)), torch.zeros(10, 2, device="cuda")),
           lambda: nomad.route_gradient(x[:, :4], r._replace(experts=none.int()), torch.zeros(10, 2, device="cuda")), lambda: nomad.grouped_product(line, w, offsets),
           lambda: nomad.grouped_product(x, w, offsets, slope_at=none), lambda: nomad.grouped_product(x, w, offsets, slope_at=line), lambda: nomad.grouped_product(x, w, none.int()),
           lambda: nomad.grouped_product(x, w, offsets, activation=["silu"]), lambda: nomad.grouped_product(x, w, offsets, activation=2),
           lambda: nomad.grouped_product(x, w, offsets, order=order, per_row=2 ** 31), lambda: nomad.grouped_weight_gradient(x, x, offsets, order=order, per_row=2 ** 40),
           lambda: nomad.grouped_weight_gradient(none, x, offsets), lambda: nomad.combine(x, r.slots.view(-1)), lambda: nomad.combine(x, none.int()),
           lambda: nomad.combine_gradient(none, x, r.slots), lambda: nomad.combine_gradient(line, x, r.slots), lambda: nomad.combine_gradient(x, x, r.slots.view(-1))]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            note(f"refusal {i} did not happen")
    assert nomad.grouped_product(x, w, offsets, per_row=2 ** 40).shape == (10, 4)     # (no order: not looked at)
