"""The learned map's oracle against differences and cases worked by hand (no GPU)."""
import numpy as np
import pytest

from oracle import map_oracle as mo


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[at] += h
        down[at] -= h
        g[at] = (f(up) - f(down)) / (2 * h)
    return g


def test_routing_by_hand():
    inf = float("inf")
    logits = np.array([[1.0, 3.0, 3.0, 0.0], [-inf, -inf, -inf, -inf], [float("nan"), 2.0, -inf, 2.0], [0.0, -0.0, -1.0, -inf]])
    experts, weights, offsets, order, slots = mo.route(logits, 2)
    assert experts.tolist() == [[1, 2], [-1, -1], [1, 3], [0, 1]]
    assert np.allclose(weights, [[0.5, 0.5], [0, 0], [0.5, 0.5], [0.5, 0.5]])
    assert offsets.tolist() == [0, 1, 4, 5, 6]
    assert order.tolist() == [6, 0, 4, 7, 1, 5, -1, -1]
    assert slots.tolist() == [[1, 4], [-1, -1], [2, 5], [0, 3]]
    _, full, _, _, _ = mo.route(logits, 1, normalize=False)
    e = np.exp([1.0, 3.0, 3.0, 0.0])
    assert np.isclose(full[0, 0], e[1] / e.sum()) and np.isclose(full[2, 0], 0.5)


@pytest.mark.parametrize("normalize", [True, False])
def test_route_gradient_against_differences(normalize):
    rng = np.random.default_rng(3)
    logits, c = rng.normal(size=(5, 7)), rng.normal(size=(5, 3))
    experts, weights, *_ = mo.route(logits, 3, normalize)
    got = mo.route_gradient(logits, experts, weights, c, normalize)
    want = _difference(lambda l: float((mo.route(l, 3, normalize)[1] * c).sum()), logits)
    assert np.abs(got - want).max() < 1e-8


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_slopes_against_differences(name):
    z = np.array([-6.0, -1.3, -0.2, 0.3, 1.7, 8.0])
    want = (mo.act(z + 1e-6, name) - mo.act(z - 1e-6, name)) / 2e-6
    assert np.abs(mo.slope(z, name) - want).max() < 1e-8


def test_layer_gradients_against_differences():
    rng = np.random.default_rng(4)
    n, k, groups, d, h, o = 6, 2, 3, 4, 5, 2
    logits = rng.normal(size=(n, groups))
    logits[2] = -np.inf                                        # a row without experts
    experts, weights, offsets, order, slots = mo.route(logits, k)
    x, w1, b1 = rng.normal(size=(n, d)), rng.normal(size=(groups, h, d)), rng.normal(size=(groups, h))
    w2, c = rng.normal(size=(groups, o, h)), rng.normal(size=(n, o))

    def loss(x, w1, b1, w2):
        hid, _, _ = mo.product(x, w1, offsets, b1, "silu", order, k)
        return float((mo.combine(mo.product(hid, w2, offsets)[0], slots, weights) * c).sum())
    hid, z, _ = mo.product(x, w1, offsets, b1, "silu", order, k)
    out = mo.product(hid, w2, offsets)[0]
    do, dweights = mo.combine_gradient(c, out, slots, weights)
    dw2, _, _, _ = mo.weight_gradient(do, hid, offsets)
    dz = mo.product(do, w2.transpose(0, 2, 1), offsets, None, "silu", slope_at=z)[0]
    dw1, db1, _, _ = mo.weight_gradient(dz, x, offsets, order, k)
    dx = mo.combine(mo.product(dz, w1.transpose(0, 2, 1), offsets)[0], slots)
    for got, at, f in ((dx, x, lambda v: loss(v, w1, b1, w2)), (dw1, w1, lambda v: loss(x, v, b1, w2)), (db1, b1, lambda v: loss(x, w1, v, w2)),
                       (dw2, w2, lambda v: loss(x, w1, b1, v))):
        assert np.abs(got - _difference(f, at)).max() < 1e-7
    dl = _difference(lambda l: float((mo.combine(out, slots, mo.route(l, k)[1]) * c).sum()), np.where(np.isinf(logits), 0.0, logits))
    got = mo.route_gradient(logits, experts, weights, dweights)
    assert np.abs(got - dl)[[0, 1, 3, 4, 5]].max() < 1e-7 and (got[2] == 0).all()


def test_adamw_first_step_is_the_sign():
    p, m, v = mo.adamw(np.array([1.0, -2.0]), np.array([0.5, -3.0]), np.zeros(2), np.zeros(2), 1, 0.1, 0.9, 0.999, 0.0, 0.0)
    assert np.allclose(p, [0.9, -1.9]) and np.allclose(m, [0.05, -0.3]) and np.allclose(v, [2.5e-4, 9e-3])
    assert np.allclose(mo.adamw(np.array([1.0]), np.zeros(1), np.zeros(1), np.zeros(1), 1, 0.1, 0.9, 0.999, 1e-8, 0.5)[0], 0.95)


def test_draws_are_philox_and_even():
    from oracle import c_oracle
    rng = np.random.default_rng(6)
    for _ in range(20):
        counter, key = rng.integers(0, 2 ** 32, size=4), rng.integers(0, 2 ** 32, size=2)
        assert mo.philox(counter, key).tolist() == list(c_oracle.philox(counter.tolist(), key.tolist()))
    u = mo.draws(100_003, 12345, True)
    assert u.shape == (100_003,) and u.min() > 0 and u.max() < 1
    assert abs(u.mean() - 0.5) < 6 / np.sqrt(12 * u.size) and (mo.draws(100_003, 12346, True) != u).mean() > 0.99
    words = mo.philox([[2, 0, 0, 0]], (7, 0))[0]
    assert mo.draws(24, 7, False)[16:20].tolist() == [(int(w) + 0.5) / 65536 for w in (words[0] & np.uint64(65535), words[0] >> np.uint64(16), words[1] & np.uint64(65535), words[1] >> np.uint64(16))]


def test_dithered_averages_follow_changing_gradients():
    """beta2 = 0.999, half of each block's gradients shrinking to 3 % after 1,000 of 5,000 steps.  A code's draw is right in expectation and the
    average linear, so the decoded average is off by noise alone: a step's change of v by no more than 0.001 v is drawn from two codes whose
    values are 4 / c + 6 / c^2 of v apart, a variance of no more than their product, and earlier noise decays no slower than v does."""
    blocks, steps, beta2 = 4, 5000, 0.999
    n = blocks * 256
    small = np.arange(n) % 2 == 1
    codes, scales, exact = np.zeros(n), np.zeros(blocks), np.zeros(n)
    variance = 0.0
    for step in range(1, steps + 1):
        g = np.where(small & (step > 1000), 0.03, 1.0)
        v = beta2 * mo.decode_second(codes, scales) + (1 - beta2) * g * g
        exact = beta2 * exact + (1 - beta2) * g * g
        codes, scales, _ = mo.encode_second(v, mo.draws(n, step, True))
        c = 255.0 * (exact[1] / exact[0]) ** 0.25
        variance += (1 - beta2) * (4 / c + 6 / c ** 2)
    got = mo.decode_second(codes, scales)
    assert abs(got[small].mean() / exact[1] - 1) < 6 * np.sqrt(variance / small.sum())
    assert np.abs(got[~small] / exact[0] - 1).max() < 1e-6      # the largest of their blocks: code 255, no noise
    assert np.sqrt(exact[1]) < 0.15 * np.sqrt(exact[0])         # (and they have become small)


def test_codes_of_8_bits_are_the_nearest_at_any_scale():
    """Every code lies between its borders, and the value it stands for within half a step, for scales from one to the smallest."""
    rng = np.random.default_rng(5)
    for top in (1.0, 1e-20, 1e-28, 1.2e-29, 1e-33, 4e-35, 1e-37, 2.0 ** -126):
        x = rng.normal(size=700) * 10.0 ** rng.uniform(-6, 0, size=700)
        x *= top / np.abs(x).max()
        x[[0, 300, 600]] = top, -top, top                     # every block has that scale
        for encode, decode, v, most, power in ((mo.encode_first, mo.decode_first, x, 127, 2), (mo.encode_second, mo.decode_second, np.abs(x), 255, 4)):
            codes, scales, t = encode(v)
            assert all(scales[b] == np.abs(v[256 * b:256 * b + 256]).max() for b in range(3)) and np.abs(codes).max() == most
            a = np.abs(codes)
            assert np.all(t < (a + 0.5) ** power * (1 + 1e-12)) and np.all((t >= np.maximum(a - 0.5, 0.0) ** power * (1 - 1e-12)) | ((power == 4) & (a == 1)))
            value = decode(codes, scales)
            assert np.all(np.abs(np.abs(value) - np.abs(v)) <= top * ((a + 0.5) ** power - np.maximum(a - 0.5, 0.0) ** power) / most ** power)
            assert np.all((np.sign(value) == np.sign(v)) | (codes == 0))
    assert (mo.encode_first(np.full(10, 1e-38))[0] == 0).all() and (mo.encode_second(np.zeros(10))[0] == 0).all()
