"""Routing by scores, dense products and the gradients' norm against the float64 oracle, at the sizes, layouts and masks where they can go
wrong.

Tolerances are bounds: a float32 sum of K terms in any order is off by at most (K + 8) 2^-24 times the sum of their absolute
values; an activation passes that on with a slope of at most 1.13 and adds its own rounding, a few units of 2^-24 times (1 + |z|) |z| where the
result is float32 and 2^-16 of itself where it is not; a residual is added with one rounding, and the result is rounded once to its
type."""
import math

import numpy as np
import pytest
import torch

import paper_2505_15511_amd as nomad
from oracle import map_oracle as mo
from paper_2505_15511_amd import NomadError
from test_gpu_map_operators import BF16, F16, F32, U32, UNIT, host, near, note, randn

pytestmark = pytest.mark.gpu


# ---- routing by scores

#: n, experts, k, groups, top_groups, group_best, score, bias, type
ROUTES = [(1, 256, 8, 8, 4, 2, "sigmoid", True, F32), (1, 1, 1, 1, 1, 1, "softmax", True, F32), (7, 10, 2, 5, 2, 1, "sigmoid", False, BF16), (64, 50, 3, 5, 2, 2, "softmax", True, F16),
          (300, 64, 4, 8, 3, 2, "sigmoid", True, BF16), (1100, 256, 8, 8, 4, 2, "sigmoid", True, BF16), (1500, 50, 5, 10, 7, 1, "softmax", False, F32), (700, 1000, 3, 1, 1, 1, "softmax", True, F16),
          (400, 1024, 8, 64, 5, 2, "sigmoid", True, F32), (3000, 8, 2, 1, 1, 1, "sigmoid", True, F32), (260, 1029, 5, 3, 2, 2, "softmax", False, F32), (40, 16384, 2, 32, 1, 1, "sigmoid", True, BF16),
          (2000, 33, 1, 11, 1, 2, "softmax", True, F32), (600, 128, 2, 64, 9, 1, "sigmoid", True, F16), (500, 520, 6, 13, 6, 2, "sigmoid", False, F32), (1300, 192, 8, 16, 2, 2, "softmax", True, BF16),
          (5, 16384, 8, 1, 1, 1, "softmax", True, F32), (900, 60, 7, 4, 4, 2, "sigmoid", True, F32), (1025, 24, 2, 3, 1, 2, "sigmoid", True, F32)]


def check_scored(logits, k, bias=None, **call):
    """Exact integers; weights within a few units each and one for every term of a sum."""
    r = nomad.route_scored(logits, k, bias=bias, **call)
    experts, weights, offsets, order, slots = mo.route_scored(host(logits), k, bias=None if bias is None else bias.cpu().numpy(), **call)
    for name, got, want in (("experts", r.experts, experts), ("offsets", r.offsets, offsets), ("order", r.order, order), ("slots", r.slots, slots)):
        assert np.array_equal(got.cpu().numpy(), want), name
    assert np.array_equal(np.isnan(host(r.weights)), np.isnan(weights))
    terms = k if call.get("normalize", True) or call.get("score") == "sigmoid" else logits.shape[1]
    # (softmax shares come of differences of logits, whose rounding an exponential passes on: 2^-24 of the difference; scores are factors of up to four
    # exponentials and sums)
    spread = np.nan_to_num(np.abs(host(logits)), nan=0.0, posinf=0.0, neginf=0.0).clip(max=120.0).max() if logits.numel() else 0.0
    near(torch.nan_to_num(r.weights), np.nan_to_num(weights), (terms + 24 + 2 * spread) * U32 * np.abs(np.nan_to_num(weights)), F32, "weights")
    return r, weights


def logits_of(n, experts, rng, masks=True):
    x = (1.5 * rng.normal(size=(n, experts))).astype(np.float32)
    if masks:
        x[rng.random((n, experts)) < 0.2] = -np.inf                       # masked experts
        x[rng.random((n, experts)) < 0.05] = np.nan
        x[rng.random((n, experts)) < 0.2] = 0.5                           # ties
        x[rng.random((n, experts)) < 0.05] = -0.0
        x[rng.random((n, experts)) < 0.05] = 0.0
        x[rng.random(n) < 0.1] = -np.inf                                  # rows without any
        x[rng.random(n) < 0.1, :(experts + 1) // 2] = -np.inf             # half of the groups without any
    return x


@pytest.mark.parametrize("n,experts,k,groups,top,best,score,biased,dtype", ROUTES)
@pytest.mark.parametrize("normalize", [True, False])
def test_routing_by_scores(n, experts, k, groups, top, best, score, biased, dtype, normalize):
    note(f"scored n={n} E={experts} k={k} {groups}/{top}/{best} {score} {biased} {dtype} {normalize}")
    rng = np.random.default_rng(n + experts)
    logits = torch.from_numpy(logits_of(n, experts, rng)).to("cuda", dtype)
    bias = torch.from_numpy((0.05 * rng.normal(size=experts)).astype(np.float32)).cuda() if biased else None
    if biased and experts > 4:
        bias[::3] = 0.25                                                  # the same for many: equal logits are ties
    call = dict(score=score, normalize=normalize, scale=2.5)
    r, weights = check_scored(logits, k, bias, groups=groups, top_groups=top, group_best=best, **call)
    dw = torch.from_numpy(rng.normal(size=(n, k)).astype(np.float32)).cuda()
    got = nomad.route_scored_gradient(logits, r, dw, **call)
    want = mo.route_scored_gradient(host(logits), r.experts.cpu().numpy(), weights, host(dw), **call)
    near(got, want, 2.5 * k * np.abs(host(dw)).max() * (experts + 32) * U32, dtype, "dlogits")


@pytest.mark.parametrize("groups,top,best", [(1, 1, 1), (8, 3, 2), (8, 3, 1)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_sums_that_32_bits_cannot_tell_apart(groups, top, best, score):
    """Biases that lift every expert to the same sum but for what is left of their rounding: 64 bits say which is larger."""
    note(f"near ties {groups} {score}")
    rng = np.random.default_rng(17)
    base = rng.normal(size=64)
    s = 1.0 / (1.0 + np.exp(-base.astype(np.float32).astype(np.float64))) if score == "sigmoid" else np.exp(base) / np.exp(base).sum()
    bias = torch.from_numpy((1.0 - s).astype(np.float32)).cuda()
    x = np.repeat(base[None].astype(np.float32), 1200, 0)
    x += (1e-6 * rng.normal(size=x.shape)).astype(np.float32) * (rng.random(x.shape) < 0.5)
    check_scored(torch.from_numpy(x).cuda(), 4, bias, groups=groups, top_groups=top, group_best=best, score=score)
    zeros = torch.zeros(700, 64, device="cuda")                           # and rows of nothing but ties
    check_scored(zeros, 4, torch.zeros(64, device="cuda"), groups=groups, top_groups=top, group_best=best, score=score)


def test_scored_strides_and_extremes():
    note("scored strides and extremes")
    rng = np.random.default_rng(1)
    base = torch.from_numpy(rng.normal(size=(900, 70)).astype(np.float32)).cuda()
    bias = torch.from_numpy((0.1 * rng.normal(size=64)).astype(np.float32)).cuda()
    grouped = dict(groups=8, top_groups=2, group_best=2)
    for score in ("sigmoid", "softmax"):
        for x in (base[:, 3:67], base[::3, :64], base[5:6].expand(600, 70)[:, :64]):
            check_scored(x, 3, bias, score=score, **grouped)              # rows apart, not aligned, one row for all
        lowest = torch.finfo(F32).min
        x = torch.full((400, 12), lowest, device="cuda")                  # a mask of the lowest number is a number
        check_scored(x, 3, None, score=score, groups=3, top_groups=2)
        check_scored(x, 3, torch.arange(12, device="cuda") * 0.01, score=score, groups=3, top_groups=2, group_best=2)
        x = 30.0 * torch.from_numpy(rng.normal(size=(500, 12)).astype(np.float32)).cuda()
        check_scored(x, 3, bias[:12].contiguous(), score=score)           # sigmoids that are all but 0 and 1
        check_scored(x - 150.0, 3, None, score=score)                     # and too small for a float
        x[7, 2] = float("inf")
        check_scored(x, 3, bias[:12].contiguous(), score=score)
        check_scored(x, 3, bias[:12].contiguous(), score=score, groups=4, top_groups=2, group_best=2)
        odd = bias[:12].clone()
        odd[1], odd[2], odd[3], odd[4], odd[5] = float("inf"), float("nan"), -float("inf"), 1e30, -1e30
        check_scored(x[100:], 3, odd, score=score)
        r = nomad.route_scored(torch.empty(0, 9, device="cuda"), 2, score=score, groups=3, top_groups=2)
        assert r.offsets.tolist() == [0] * 10 and r.order.numel() == 0 and nomad.route_scored_gradient(torch.empty(0, 9, device="cuda"), r, r.weights).shape == (0, 9)
    many = (5.0 + 1e3 * torch.rand(300, 16, device="cuda"))                # large biases: sums lose what scores differ by, in 64 bits too
    check_scored(many.neg() * 0.01, 4, 1e4 * torch.randn(16, device="cuda").round(), groups=4, top_groups=2, group_best=2)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("scale", [1.0, 2.5, 0.3])
@pytest.mark.parametrize("n,experts", [(9, 649), (37, 62), (3000, 200)])
def test_one_expert_alone_has_the_whole_weight(score, scale, n, experts):
    """Its share is 1 and does not depend on its logit: no rounding is left in either."""
    note(f"alone {score} {scale} {n} {experts}")
    rng = np.random.default_rng(n)
    logits, dw = randn((n, experts), F32, rng, 2.0), randn((n, 1), F32, rng)
    r = nomad.route_scored(logits, 1, score=score, bias=randn((experts,), F32, rng, 0.1), scale=scale)
    assert (r.weights == scale).all() and not nomad.route_scored_gradient(logits, r, dw, score=score, scale=scale).any()
    logits[::2, 1:] = -math.inf                                           # one of three places taken
    r = nomad.route_scored(logits, 3, score=score, scale=scale)
    assert (r.weights[::2, 0] == scale).all() and not r.weights[::2, 1:].any()
    assert not nomad.route_scored_gradient(logits, r, dw.expand(n, 3).contiguous(), score=score, scale=scale)[::2].any()


def test_scored_many_rows():
    """Half a million rows against sums in 64 bits: some of them need those."""
    note("scored 500000 x 128")
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn(500_000, 128, device="cuda", generator=gen)
    logits[::97] = -float("inf")
    bias = 0.02 * torch.randn(128, device="cuda", generator=gen)
    r = nomad.route_scored(logits, 2, bias=bias)
    x = logits.double()
    c = torch.where(x > -math.inf, 1.0 / (1.0 + torch.exp(-x)) + bias.double(), -math.inf)
    top = torch.sort(c, dim=1, descending=True, stable=True)
    want = torch.where(top.values[:, :2] > -float("inf"), top.indices[:, :2], -1).int()
    assert torch.equal(r.experts, want)
    flat = torch.where(want >= 0, want, 128).reshape(-1)
    by, order = torch.sort(flat, stable=True)
    assert torch.equal(r.order, torch.where(by < 128, order, -1).int())
    assert torch.equal(r.offsets.long(), torch.searchsorted(by, torch.arange(129, device="cuda")))
    assert torch.equal(r.slots.reshape(-1)[r.order[:int(r.offsets[-1])].long()], torch.arange(int(r.offsets[-1]), device="cuda").int())


@pytest.mark.parametrize("experts", [1, 7, 256, 16384])
def test_balance(experts):
    note(f"balance {experts}")
    rng = np.random.default_rng(experts)
    bias = torch.from_numpy(rng.normal(size=experts).astype(np.float32)).cuda()
    count = rng.integers(0, 5, size=experts)
    count[: experts // 2] = 2                                             # some at the mean, where it is whole
    for c in (count, np.zeros(experts, np.int64), np.full(experts, 100_000)):
        offsets = np.concatenate([[0], np.cumsum(c)]).astype(np.int32)
        got = nomad.balance_bias(bias, torch.from_numpy(offsets).cuda(), 1e-3)
        near(got, mo.balance_bias(host(bias), offsets, np.float64(np.float32(1e-3))), 0.0, F32, "bias")


def test_balance_evens_out():
    """What the bias is for: logits that favour one expert, and loads that come together."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(4096, 16, device="cuda", generator=gen)
    logits[:, 3] += 2.0
    bias = torch.zeros(16, device="cuda")
    load = lambda: torch.diff(nomad.route_scored(logits, 2, bias=bias).offsets).float()   # noqa: E731
    first = load().max().item()
    for _ in range(200):
        bias = nomad.balance_bias(bias, nomad.route_scored(logits, 2, bias=bias).offsets, 5e-3)
    note(f"  largest load {first} -> {load().max().item()} of a mean of 512")
    assert load().max().item() < first


# ---- dense products

#: (rows, in, out, type): single rows, few rows on either side of sixteens, long sums that are cut, every tile, odd sizes
DENSE = [(1, 1, 1, F32), (1, 768, 2048, BF16), (1, 50, 129, F32), (3, 4097, 40, F16), (16, 8192, 96, BF16), (17, 2056, 130, F16), (33, 512, 16, F32), (64, 1000, 72, BF16), (65, 8192, 72, BF16),
         (130, 7, 3, BF16), (300, 50, 129, F32), (500, 4096, 136, F16), (257, 2049, 2, F32), (1000, 64, 2, BF16), (700, 129, 130, F16), (2050, 264, 272, BF16), (4099, 256, 4104, BF16), (5000, 20, 12, F32),
         (0, 16, 16, BF16), (100, 1, 70, F16), (9000, 136, 2056, F16), (300, 8192, 20, F32)]


def bound_of(size, want_z, inner, dtype):
    """Of act(z): of float32 results, and of others."""
    own = 8 * U32 * (1 + np.abs(want_z)) * np.abs(want_z) + (0.0 if dtype == F32 else 2.0 ** -16 * np.abs(want_z))
    return 1.13 * (inner + 8) * U32 * size + own


@pytest.mark.parametrize("rows,inner,out,dtype", DENSE)
@pytest.mark.parametrize("turned", [False, True])
def test_dense_product(rows, inner, out, dtype, turned):
    note(f"dense rows={rows} {inner}->{out} {dtype} turned={turned}")
    rng = np.random.default_rng(rows + inner + out)
    x = randn((rows, inner), dtype, rng)
    w = randn((inner, out) if turned else (out, inner), dtype, rng, inner ** -0.5)
    w = w.t() if turned else w
    bias, residual = randn((out,), dtype, rng), randn((rows, out), dtype, rng)
    for activation in ("none", "relu", "silu", "gelu"):
        for r in (None, residual):
            y, z = nomad.dense_product(x, w, bias, activation, r, keep=True)
            assert torch.equal(y, nomad.dense_product(x, w, bias, activation, r))
            want_y, want_z, size = mo.dense(host(x), host(w), host(bias), activation, None if r is None else host(r))
            bound = (inner + 8) * U32 * size
            near(z, want_z, bound, dtype, "z")
            near(y, want_y, bound_of(size, want_z, inner, dtype) + U32 * (np.abs(want_y) + np.abs(want_z)), dtype, activation + (" + r" if r is not None else ""))
        if activation != "none":
            back = nomad.dense_product(x, w, activation=activation, slope_at=z)
            want, plain, size = mo.dense(host(x), host(w), activation=activation, slope_at=host(z))
            near(back, want, 1.13 * (inner + 8) * U32 * size + (16 * U32 * (1 + np.abs(host(z))) + (0.0 if dtype == F32 else 2.0 ** -16)) * np.abs(plain), dtype, "slope of " + activation)
    if dtype != F32:
        for activation, r in (("none", None), ("gelu", residual)):
            wide, z = nomad.dense_product(x, w, bias, activation, r, keep=True, out_dtype=F32)
            want_y, want_z, size = mo.dense(host(x), host(w), host(bias), activation, None if r is None else host(r))
            near(wide, want_y, bound_of(size, want_z, inner, F32) + U32 * (np.abs(want_y) + np.abs(want_z)), F32, "float32 results " + activation)
            near(z, want_z, (inner + 8) * U32 * size, dtype, "z")
        plain = nomad.dense_product(x, w, out_dtype=F32)
        want_y, want_z, size = mo.dense(host(x), host(w))
        near(plain, want_y, (inner + 8) * U32 * size, F32, "float32 results")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_dense_layouts(dtype):
    """Rows apart, columns off by an element, one residual row for all, and numbers that are not finite beside the operands."""
    note(f"dense layouts {dtype}")
    rng = np.random.default_rng(9)
    big, wide, rest = (torch.full(s, float("nan"), device="cuda", dtype=dtype) for s in ((310, 160), (100, 170), (310, 120)))
    for rows in (5, 260):
        for a, b, c, d, out in ((8, 136, 8, 8, 64), (1, 130, 3, 1, 67), (0, 64, 0, 16, 80), (3, 132, 1, 5, 1)):
            inner = b - a
            x, w, r = big[7:7 + rows, a:b], wide[d:d + out, c:c + inner], rest[3:3 + rows, d:d + out]
            for t in (x, w, r):
                t.copy_(randn(t.shape, dtype, rng, 0.3))
            want, _, size = mo.dense(host(x), host(w), None, "silu", host(r))
            near(nomad.dense_product(x, w, activation="silu", residual=r), want, bound_of(size, size, inner, dtype) + 2 * U32 * (np.abs(want) + size), dtype, f"{rows} rows of {a}:{b}")
            one = r[1:2].expand(rows, out)
            want, _, size = mo.dense(host(x), host(w), None, None, host(one))
            near(nomad.dense_product(x, w, residual=one), want, (inner + 8) * U32 * (size + np.abs(want)), dtype, "one row for all")
            turned = torch.full((inner + 3, out + 9), float("nan"), device="cuda", dtype=dtype)
            turned[2:2 + inner, 4:4 + out] = w.t()
            near(nomad.dense_product(x, turned[2:2 + inner, 4:4 + out].t(), residual=one), want, (inner + 8) * U32 * (size + np.abs(want)), dtype, "turned")
            dx, dw, db = nomad.dense_gradient(r, x, turned[2:2 + inner, 4:4 + out].t())
            want = mo.dense_gradient(host(r), host(x), host(w))
            near(dx, want[0], (out + 8) * U32 * (np.abs(host(r)) @ np.abs(host(w))), dtype, "dx")
            near(dw, want[1], (rows + 8) * U32 * (np.abs(host(r)).T @ np.abs(host(x))), dtype, "dw")
            near(db, want[2], (rows + 8) * U32 * np.abs(host(r)).sum(0), F32, "db")
            for t in (x, w, r):
                t.fill_(float("nan"))
    # a row with a NaN stays by itself, and so does one with an infinity
    x, w = randn((300, 72), dtype, rng), randn((40, 72), dtype, rng)
    want = nomad.dense_product(x, w, residual=w[0, :40].expand(300, 40))
    x[11, 3], x[299, 71] = float("nan"), float("inf")
    got = nomad.dense_product(x, w, residual=w[0, :40].expand(300, 40))
    assert torch.isnan(got[11]).all() and not torch.isfinite(got[299]).any()
    keep = torch.ones(300, dtype=torch.bool)
    keep[[11, 299]] = False
    assert torch.equal(got[keep.cuda()], want[keep.cuda()])


#: (rows, in, out, type)
BACK = [(1, 1, 1, F32), (1, 768, 200, BF16), (3, 50, 129, F32), (700, 129, 50, F16), (2050, 264, 272, BF16), (20_011, 50, 129, F32), (5000, 256, 2, F32), (9000, 8, 1030, BF16), (0, 24, 16, F16),
        (33_000, 72, 136, BF16), (257, 2048, 40, BF16), (130, 16, 16, F16), (4100, 4104, 264, BF16), (2000, 3, 4112, F16)]


@pytest.mark.parametrize("rows,inner,out,dtype", BACK)
@pytest.mark.parametrize("activation", [None, "silu", "gelu", "relu"])
def test_dense_gradient(rows, inner, out, dtype, activation):
    note(f"dense gradient rows={rows} {inner}->{out} {dtype} {activation}")
    rng = np.random.default_rng(rows + inner + out)
    x, dy, w = randn((rows, inner), dtype, rng), randn((rows, out), dtype, rng), randn((out, inner), dtype, rng, inner ** -0.5)
    z = randn((rows, out), dtype, rng, 2.0) if activation else None
    want_dx, want_dw, want_db, dz = mo.dense_gradient(host(dy), host(x), host(w), activation, None if z is None else host(z))
    # the slope's own error, and dz rounded to the operands' type before the products (its sums are not)
    slope = 0.0 if z is None else (16 * U32 * (1 + np.abs(host(z))) + (0.0 if dtype == F32 else 2.0 ** -16)) * np.abs(host(dy))
    off = slope + (UNIT[dtype] * np.abs(dz) + (2.0 ** -25 if dtype == F16 else 0.0) if z is not None else 0.0)
    off = off + np.zeros_like(dz)
    for turned in (False, True):
        ww = w.t().contiguous().t() if turned else w
        dx, dw, db = nomad.dense_gradient(dy, x, ww, activation, z)
        near(dx, want_dx, (out + 8) * U32 * (np.abs(dz) @ np.abs(host(w))) + 1.01 * off @ np.abs(host(w)), dtype, "dx")
        near(dw, want_dw, (rows + 8) * U32 * (np.abs(dz).T @ np.abs(host(x))) + 1.01 * off.T @ np.abs(host(x)), dtype, "dw")
        near(db, want_db, (rows + 8) * U32 * np.abs(dz).sum(0) + (slope + np.zeros_like(dz)).sum(0), F32, "db")
    wide = nomad.dense_gradient(dy, x, w, activation, z, out_dtype=F32)
    near(wide[1], want_dw, (rows + 8) * U32 * (np.abs(dz).T @ np.abs(host(x))) + 1.01 * off.T @ np.abs(host(x)), F32, "dw in float32")
    again = nomad.dense_gradient(dy, x, w, activation, z, out_dtype=F32)
    assert all(torch.equal(a, b) for a, b in zip(wide, again))            # sums meet in one order
    only = nomad.dense_gradient(dy, x, w, activation, z, need_dx=False, bias=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], nomad.dense_gradient(dy, x, w, activation, z)[1])
    only = nomad.dense_gradient(dy, x, w, activation, z, need_dw=False)
    assert only[1] is None and only[2] is None and torch.equal(only[0], wide[0])


def test_dense_gradient_against_differences():
    """A layer with its residual, as a function, along random directions: float32 differences of second order over a step of 2^-6 are good to some
    2^-12 (the third derivative of GELU times the step's square) and their own roundings."""
    rng = np.random.default_rng(12)
    x, w, b, c = randn((200, 24), F32, rng), randn((40, 24), F32, rng, 0.2), randn((40,), F32, rng), randn((200, 40), F32, rng)
    r = randn((200, 40), F32, rng)
    y, z = nomad.dense_product(x, w, b, "gelu", r, keep=True)
    dx, dw, db = nomad.dense_gradient(c, x, w, "gelu", z)
    loss = lambda x, w, b, r: (nomad.dense_product(x, w, b, "gelu", r).double() * c.double()).sum().item()   # noqa: E731
    h = 2.0 ** -6
    for i, (value, grad) in enumerate(((x, dx), (w, dw), (b, db), (r, c))):
        d = randn(value.shape, F32, rng)
        d /= d.norm()
        at = lambda s: loss(*[v + s * d if j == i else v for j, v in enumerate((x, w, b, r))])   # noqa: E731
        difference, formula = (at(h) - at(-h)) / (2 * h), (grad.double() * d.double()).sum().item()
        scale = grad.double().norm().item()
        note(f"  {difference} {formula} of {scale}")
        assert abs(difference - formula) <= 2.0 ** -9 * scale


@pytest.mark.parametrize("rows,inner,out,dtype", [(12_000, 768, 2048, BF16), (16_500, 1032, 512, F16), (70_001, 264, 512, BF16)])
def test_large_tiles_with_sums_in_parts(rows, inner, out, dtype):
    """Against products in 64 bits on the GPU."""
    note(f"large tiles {rows} {inner}->{out} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dy, w = (torch.randn(s, device="cuda", generator=gen).to(dtype) for s in ((rows, inner), (rows, out), (out, inner)))
    dx, dw, db = nomad.dense_gradient(dy, x, w)
    wide = nomad.dense_gradient(dy, x, w, out_dtype=F32, need_dx=False)
    a, b, c = dy.double(), x.double(), w.double()
    near(dx, host(a @ c), (out + 8) * U32 * host(a.abs() @ c.abs()), dtype, "dx")
    near(dw, host(a.t() @ b), (rows + 8) * U32 * host(a.abs().t() @ b.abs()), dtype, "dw")
    near(wide[1], host(a.t() @ b), (rows + 8) * U32 * host(a.abs().t() @ b.abs()), F32, "dw in float32")
    near(db, host(a.sum(0)), (rows + 8) * U32 * host(a.abs().sum(0)), F32, "db")
    r = dy[:64, :out]
    near(nomad.dense_product(x[:64], w, residual=r), host(b[:64] @ c.t() + r.double()), (inner + 8) * U32 * host(b[:64].abs() @ c.abs().t() + r.double().abs()), dtype, "few rows")


def test_places_that_pass_32_bits():
    """More than 2^32 elements of an operand, a residual, gradients and logits: the last rows are as they are by themselves."""
    note("beyond 32 bits")
    n = 34_000_000
    x = torch.zeros(n, 128, device="cuda", dtype=BF16)
    tail = torch.randn(1000, 128, device="cuda").to(BF16)
    x[-1000:] = tail
    w = torch.randn(128, 128, device="cuda").to(BF16)
    y = nomad.dense_product(x, w, activation="silu", residual=x)
    want = (torch.nn.functional.silu(tail.double() @ w.double().t()) + tail.double())
    bound = host(tail.double().abs() @ w.double().abs().t())
    near(y[-1000:], host(want), 1.13 * 136 * U32 * bound + (8 * U32 * (1 + bound) + 2.0 ** -16) * bound + 2 * U32 * host(want.abs()), BF16, "product")
    assert not y[:-1000:9973].any()
    del y
    dx, dw, db = nomad.dense_gradient(x, x, w)
    near(dx[-1000:], host(tail.double() @ w.double()), 136 * U32 * host(tail.double().abs() @ w.double().abs()), BF16, "dx")
    near(dw, host(tail.double().t() @ tail.double()), 1008 * U32 * host(tail.double().abs().t() @ tail.double().abs()), BF16, "dw")
    near(db, host(tail.double().sum(0)), 1008 * U32 * host(tail.double().abs().sum(0)), F32, "db")
    del dx
    norm, _ = nomad.gradient_norm([x, tail])
    full = math.sqrt(2.0) * tail.double().norm().item()
    assert abs(norm.item() - full) <= 1.01 * U32 * full
    bias = 0.1 * torch.randn(128, device="cuda")
    call = dict(groups=8, top_groups=3, group_best=2)
    r = nomad.route_scored(x, 2, bias=bias, **call)
    alone = nomad.route_scored(tail, 2, bias=bias, **call)
    assert torch.equal(r.experts[-1000:], alone.experts) and torch.equal(r.weights[-1000:], alone.weights)
    assert int(r.offsets[-1]) == 2 * n and torch.equal(r.order[r.slots[-1000:].reshape(-1).long()], torch.arange(2 * n - 2000, 2 * n, device="cuda").int())
    dw = torch.zeros(n, 2, device="cuda")
    dw[-1000:] = torch.randn(1000, 2, device="cuda")
    got = nomad.route_scored_gradient(x, r, dw)
    assert torch.equal(got[-1000:], nomad.route_scored_gradient(tail, alone, dw[-1000:].contiguous())) and not got[:-1000:9973].any()


# ---- the gradients' norm

@pytest.mark.parametrize("count,largest", [(1, 1), (1, 100_003), (5, 4097), (200, 3000), (400, 9), (3, 9_000_001)])
def test_norm(count, largest):
    """Sums are in 64 bits: one rounding of the result."""
    note(f"norm {count} {largest}")
    gen = torch.Generator().manual_seed(count + largest)
    types, grads = (F32, BF16, F16), []
    for i in range(count):
        n = max(0, largest // (1 + i % 7) - i % 3)
        held = torch.randn(n + 3, generator=gen).mul_(10.0 ** (i % 5 - 2)).to("cuda", types[i % 3])
        grads.append(held[i % 3:i % 3 + n])                                # beginning anywhere
    grads[0] = grads[0].reshape(-1, 1)
    norm, scale = nomad.gradient_norm(grads)
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    assert norm.shape == scale.shape == (1,) and abs(norm.item() - want) <= 1.01 * U32 * want and scale.item() == 1.0
    for factor in (None, 0.125, -3.0):
        given = None if factor is None else torch.tensor([factor], device="cuda")
        for most in (0.0, 0.3 * want, 2.0 * want, 7.0 * want, math.inf):
            norm, scale = nomad.gradient_norm(grads, most, given)
            full = want * abs(factor or 1.0)
            rate = (factor or 1.0) * (1.0 if full <= most else most / full)
            assert abs(norm.item() - full) <= 1.01 * U32 * full and abs(scale.item() - rate) <= 1.01 * U32 * abs(rate)
    assert all(torch.equal(a, b) for a, b in zip(nomad.gradient_norm(grads, 1.0), nomad.gradient_norm(grads, 1.0)))


def test_norm_extremes():
    note("norm extremes")
    for value, want in ((1e-30, 1e-30 * math.sqrt(1000)), (1e30, 1e30 * math.sqrt(1000)), (2.0 ** -149, 2.0 ** -149 * math.sqrt(1000))):
        norm, scale = nomad.gradient_norm([torch.full((1000,), value, device="cuda")], want / 2)
        assert abs(norm.item() - want) <= 1e-6 * want + 2.0 ** -149
        assert abs(scale.item() - 0.5) < 1e-6 or value < 1e-44                # (a value of one unit is off by its rounding)
    norm, scale = nomad.gradient_norm([torch.full((4,), 3e38, device="cuda")], 1.0)
    assert norm.item() == math.inf and abs(scale.item() - 1 / 6e38) < 1e-44  # the norm passes float32, the factor does not
    none = torch.empty(0, device="cuda")
    assert [t.item() for t in nomad.gradient_norm([none, none], 1.0)] == [0.0, 1.0]
    g = torch.ones(5000, device="cuda")
    g[4321] = float("nan")
    assert all(math.isnan(t.item()) for t in nomad.gradient_norm([g], 1.0))
    g[4321] = -float("inf")
    norm, scale = nomad.gradient_norm([g], 1.0)
    assert norm.item() == math.inf and scale.item() == 0.0
    assert nomad.gradient_norm([g])[1].item() == 1.0


# ---- together

def a_step(x, logits, bias, layers, target, limit, stream=None):
    """A shared layer with the routed experts' sum as its residual, every gradient, and the norm: as a fitting step would."""
    w, b, w1, w2 = layers
    r = nomad.route_scored(logits, 3, bias=bias, groups=4, top_groups=2, group_best=2, scale=1.5, stream=stream)
    h, z = nomad.grouped_product(x, w1, r.offsets, activation="silu", order=r.order, per_row=3, keep=True, stream=stream)
    o = nomad.grouped_product(h, w2, r.offsets, stream=stream)
    y, zs = nomad.dense_product(x, w, b, "gelu", residual=nomad.combine(o, r.slots, r.weights, stream=stream), keep=True, stream=stream)
    dy = y - target if stream is None else target
    dx, dw, db = nomad.dense_gradient(dy, x, w, "gelu", zs, stream=stream)
    do, dweights = nomad.combine_gradient(dy, o, r.slots, r.weights, order=r.order, stream=stream)
    dw2, _ = nomad.grouped_weight_gradient(do, h, r.offsets, bias=False, stream=stream)
    dz = nomad.grouped_product(do, w2.transpose(1, 2), r.offsets, activation="silu", slope_at=z, stream=stream)
    dw1, _ = nomad.grouped_weight_gradient(dz, x, r.offsets, order=r.order, per_row=3, bias=False, stream=stream)
    dlogits = nomad.route_scored_gradient(logits, r, dweights, scale=1.5, stream=stream)
    norm, scale = nomad.gradient_norm([dw, db, dw1, dw2, dlogits], limit, stream=stream)
    return y, dx, dw, db, dw1, dw2, dlogits, nomad.balance_bias(bias, r.offsets, 0.01, stream=stream), norm, scale


def made(rng, n=600):
    layers = (randn((24, 40), F32, rng, 0.2), randn((24,), F32, rng), randn((16, 32, 40), F32, rng, 0.2), randn((16, 24, 32), F32, rng, 0.2))
    return randn((n, 40), F32, rng), randn((n, 16), F32, rng), randn((16,), F32, rng, 0.05), layers, randn((n, 24), F32, rng)


def test_together():
    note("together")
    rng = np.random.default_rng(40)
    x, logits, bias, layers, target = made(rng)
    w, b, w1, w2 = (host(t) for t in layers)
    got = a_step(x, logits, bias, layers, target, 0.5)
    experts, weights, offsets, order, slots = mo.route_scored(host(logits), 3, bias=bias.cpu().numpy(), groups=4, top_groups=2, group_best=2, scale=1.5)
    h, z, _ = mo.product(host(x), w1, offsets, None, "silu", order, 3)
    o = mo.product(h, w2, offsets)[0]
    y, zs, _ = mo.dense(host(x), w, b, "gelu", mo.combine(o, slots, weights))
    dy = y - host(target)
    dx, dw, db, _ = mo.dense_gradient(dy, host(x), w, "gelu", zs)
    do, dweights = np.zeros_like(o), np.zeros_like(weights)
    for i, j in np.argwhere(slots >= 0):
        do[slots[i, j]] = weights[i, j] * dy[i]
        dweights[i, j] = dy[i] @ o[slots[i, j]]
    dw2 = mo.weight_gradient(do, h, offsets)[0]
    dz = mo.product(do, np.swapaxes(w2, 1, 2), offsets, None, "silu", slope_at=z)[0]
    dw1 = mo.weight_gradient(dz, host(x), offsets, order, 3)[0]
    dlogits = mo.route_scored_gradient(host(logits), experts, weights, dweights, scale=1.5)
    norm, scale = mo.gradient_norm([dw, db, dw1, dw2, dlogits], 0.5)
    want = (y, dx, dw, db, dw1, dw2, dlogits, mo.balance_bias(host(bias), offsets, np.float64(np.float32(0.01))), np.array([norm]), np.array([scale]))
    # a chain of six products of at most 600 terms: each is good to (600 + 8) units of its absolute sum, whose ratio to the results' size is
    # some tens here; relative to the largest result
    for name, g, v in zip(("y", "dx", "dw", "db", "dw1", "dw2", "dlogits", "bias", "norm", "scale"), got, want):
        off = np.abs(host(g) - v).max() / np.abs(v).max()
        note(f"  {name} {off:.1e}")
        assert off < 608 * 2.0 ** -24 * 6


def test_another_stream_and_graphs():
    """On another stream, in a graph that is replayed with new inputs, and in two graphs in turn."""
    note("streams and graphs")
    rng = np.random.default_rng(41)
    x, logits, bias, layers, target = made(rng, 1500)
    want = a_step(x, logits, bias, layers, target, 0.5, torch.cuda.current_stream().cuda_stream)
    side = torch.cuda.Stream()
    got = a_step(x, logits, bias, layers, target, 0.5, side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graphs = []
    for limit in (0.5, 2.0):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = a_step(x, logits, bias, layers, target, limit)
        graphs.append((graph, limit, held))
    for seed in (1, 2, 3):
        logits.copy_(torch.randn(logits.shape, generator=torch.Generator().manual_seed(seed)))
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(10 + seed)))
        for graph, limit, held in graphs:
            graph.replay()
            torch.cuda.synchronize()
            fresh = a_step(x, logits, bias, layers, target, limit)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, fresh))


def test_calls_at_once():
    """Calls on two streams that run side by side, many of them, have nothing in common."""
    note("calls at once")
    rng = np.random.default_rng(43)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    inputs = []
    for i in range(2):
        x, w, r = randn((400, 4096), BF16, rng), randn((136, 4096), BF16, rng, 0.02), randn((400, 136), BF16, rng)
        inputs.append((x, w, r, randn((5000, 128), F32, rng), randn((128,), F32, rng, 0.05)))

    def calls(x, w, r, logits, bias, stream):
        routing = nomad.route_scored(logits, 4, bias=bias, groups=8, top_groups=3, group_best=2, stream=stream)
        return (nomad.dense_product(x, w, activation="gelu", residual=r, stream=stream), *nomad.dense_gradient(r, x, w, "silu", r, stream=stream), *routing,
                nomad.route_scored_gradient(logits, routing, routing.weights, stream=stream), *nomad.gradient_norm([x, w, r, logits], 1.0, stream=stream))
    want = [calls(*each, None) for each in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(sides[i]):
                got[i].append(calls(*inputs[i], None))
    torch.cuda.synchronize()
    for i in range(2):
        for each in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(each, want[i]))


def test_clipped_step():
    """The factor goes into the step as it is: the same as gradients that were multiplied by it."""
    rng = np.random.default_rng(42)
    grads = [randn((300, 7), F32, rng), randn((11,), F32, rng)]
    norm, scale = nomad.gradient_norm(grads, 0.25)
    a, b = [torch.ones(300, 7, device="cuda"), torch.ones(11, device="cuda")], [torch.ones(300, 7, device="cuda"), torch.ones(11, device="cuda")]
    for params, g, s in ((a, grads, scale), (b, [v * scale for v in grads], None)):
        states = [nomad.adamw_state(p) for p in params]
        nomad.adamw_step(params, g, [v[0] for v in states], [v[1] for v in states], 1, grad_scale=s)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals():
    note("refusals")
    x, w, logits = torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(10, 12, device="cuda")
    y, none, line, bias = torch.zeros(10, 4, device="cuda"), torch.zeros((), device="cuda"), torch.zeros(10, device="cuda"), torch.zeros(12, device="cuda")
    r = nomad.route_scored(logits, 2)
    dw = torch.zeros(10, 2, device="cuda")
    one = torch.ones(1, device="cuda")
    bad = [lambda: nomad.route_scored(logits, 0), lambda: nomad.route_scored(logits, 13), lambda: nomad.route_scored(logits, 9), lambda: nomad.route_scored(logits.double(), 2),
           lambda: nomad.route_scored(logits.cpu(), 2), lambda: nomad.route_scored(logits.t(), 2), lambda: nomad.route_scored(line, 2), lambda: nomad.route_scored(none, 1),
           lambda: nomad.route_scored(logits, 2, score="tanh"), lambda: nomad.route_scored(logits, 2, score=1), lambda: nomad.route_scored(logits, 2, groups=5), lambda: nomad.route_scored(logits, 2, groups=0),
           lambda: nomad.route_scored(logits, 2, groups=4, top_groups=5), lambda: nomad.route_scored(logits, 2, top_groups=0), lambda: nomad.route_scored(logits, 4, groups=4, top_groups=1),
           lambda: nomad.route_scored(logits, 2, group_best=3), lambda: nomad.route_scored(logits, 2, bias=bias[:11]), lambda: nomad.route_scored(logits, 2, bias=bias.half()),
           lambda: nomad.route_scored(logits, 2, bias=bias.cpu()), lambda: nomad.route_scored(logits, 2, scale=0.0), lambda: nomad.route_scored(logits, 2, scale=float("nan")),
           lambda: nomad.route_scored(logits, 2, scale=1e39), lambda: nomad.route_scored(torch.zeros(2, 130, device="cuda"), 2, groups=65),
           lambda: nomad.route_scored_gradient(logits, r, dw[:, :1]), lambda: nomad.route_scored_gradient(logits, r, dw.double()), lambda: nomad.route_scored_gradient(logits, r._replace(experts=none.int()), dw),
           lambda: nomad.route_scored_gradient(logits[:9], r, dw), lambda: nomad.route_scored_gradient(logits, r, dw, score=None), lambda: nomad.balance_bias(bias, r.offsets[:12], 0.1),
           lambda: nomad.balance_bias(bias.double(), r.offsets, 0.1), lambda: nomad.balance_bias(none, r.offsets, 0.1), lambda: nomad.balance_bias(bias, r.offsets, float("inf")),
           lambda: nomad.balance_bias(bias.cpu(), r.offsets, 0.1),
           lambda: nomad.dense_product(x, w[:, :7]), lambda: nomad.dense_product(x, w.half()), lambda: nomad.dense_product(x, w[0]), lambda: nomad.dense_product(line, w), lambda: nomad.dense_product(x.t(), w),
           lambda: nomad.dense_product(x, torch.zeros(8, 16, device="cuda")[::2, ::2]), lambda: nomad.dense_product(x, w, bias=torch.zeros(5, device="cuda")), lambda: nomad.dense_product(x, w, bias=y),
           lambda: nomad.dense_product(x, w, activation="tanh"), lambda: nomad.dense_product(x, w, activation=["silu"]), lambda: nomad.dense_product(x, w, residual=y[:9]), lambda: nomad.dense_product(x, w, residual=none),
           lambda: nomad.dense_product(x, w, residual=y.half()), lambda: nomad.dense_product(x, w, residual=torch.zeros(4, 10, device="cuda").t()), lambda: nomad.dense_product(x, w, slope_at=y, keep=True),
           lambda: nomad.dense_product(x, w, slope_at=y, residual=y), lambda: nomad.dense_product(x, w, out_dtype=F16), lambda: nomad.dense_product(x.cpu(), w.cpu()), lambda: nomad.dense_product(x, w.cpu()),
           lambda: nomad.dense_product(x.double(), w.double()), lambda: nomad.dense_product(torch.zeros(3, 0, device="cuda"), torch.zeros(4, 0, device="cuda")),
           lambda: nomad.dense_gradient(y[:9], x, w), lambda: nomad.dense_gradient(y, x, w, "silu"), lambda: nomad.dense_gradient(y, x, w, "silu", y[:, :3]), lambda: nomad.dense_gradient(y, x, w, need_dx=False, need_dw=False),
           lambda: nomad.dense_gradient(y.half(), x, w), lambda: nomad.dense_gradient(none, x, w), lambda: nomad.dense_gradient(y, x, w, out_dtype=BF16),
           lambda: nomad.gradient_norm([]), lambda: nomad.gradient_norm([x, None]), lambda: nomad.gradient_norm([x.t()]), lambda: nomad.gradient_norm([x, x.cpu()]), lambda: nomad.gradient_norm([x.double()]),
           lambda: nomad.gradient_norm([x], -1.0), lambda: nomad.gradient_norm([x], float("nan")), lambda: nomad.gradient_norm([x], 1.0, x), lambda: nomad.gradient_norm([x], 1.0, one.double()),
           lambda: nomad.gradient_norm([x], 1.0, one.cpu())]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            note(f"refusal {i} did not happen")
    assert isinstance(NomadError(-1), RuntimeError)
