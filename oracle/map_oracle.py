"""The operators of a learned map in float64, written from their formulas (include/nomad.h): routing, products of ragged
groups with their gradients, the weighted sum, AdamW and the codes of its 8-bit states.  numpy only; nothing of the package."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256


def route(logits, k, normalize=True):
    """(experts, weights, offsets, order, slots): Python loops over rows and slots."""
    x = np.asarray(logits, dtype=np.float64)
    n, n_experts = x.shape
    experts, weights = np.full((n, k), -1, np.int32), np.zeros((n, k))
    for i in range(n):
        row = [(-x[i, e], e) for e in range(n_experts) if not math.isnan(x[i, e]) and x[i, e] > -math.inf]
        row.sort()                                            # largest first, equals by number
        chosen = row[:k]
        if not chosen:
            continue
        top = -chosen[0][0]
        among = chosen if normalize else row
        total = sum(math.exp(-v - top) for v, _ in among) if math.isfinite(top) else math.nan
        for j, (v, e) in enumerate(chosen):
            experts[i, j] = e
            weights[i, j] = math.exp(-v - top) / total if math.isfinite(top) else math.nan
    order, offsets = [], [0]
    flat = experts.reshape(-1)
    for e in range(n_experts):
        order.extend(np.flatnonzero(flat == e).tolist())
        offsets.append(len(order))
    slots = np.full(n * k, -1, np.int32)
    slots[order] = np.arange(len(order))
    order = np.array(order + [-1] * (n * k - len(order)), np.int32)
    return experts, weights, np.array(offsets, np.int32), order, slots.reshape(n, k)


def route_gradient(logits, experts, weights, dweights, normalize=True):
    x = np.asarray(logits, dtype=np.float64)
    out = np.zeros(x.shape)
    for i in range(x.shape[0]):
        there = [j for j in range(experts.shape[1]) if experts[i, j] >= 0]
        inner = sum(weights[i, j] * dweights[i, j] for j in there)
        if not there:
            continue
        if normalize:
            for j in there:
                out[i, experts[i, j]] = weights[i, j] * (dweights[i, j] - inner)
            continue
        row = np.where(np.isnan(x[i]), -math.inf, x[i])
        p = np.exp(row - row.max())
        p /= p.sum()
        given = np.zeros(x.shape[1])
        for j in there:
            given[experts[i, j]] = dweights[i, j]
        out[i] = p * (given - inner)
    return out


def erf(z):
    return np.vectorize(math.erf, otypes=[np.float64])(z)


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + erf(z / math.sqrt(2.0)))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


def rows_of(x, order, per_row, places):
    """The row of x at every place (zeros where there is none)."""
    if order is None:
        return x[:places]
    out = np.zeros((places, x.shape[1]))
    for p in range(places):
        if order[p] >= 0 and order[p] // per_row < x.shape[0]:
            out[p] = x[order[p] // per_row]
    return out


def product(x, w, offsets, bias=None, activation=None, order=None, per_row=1, slope_at=None, places=None):
    """(y, z, sum of the absolute products): zeros behind the last group."""
    places = places if places is not None else (len(order) if order is not None else x.shape[0])
    rows = rows_of(x, order, per_row, places)
    z, size = np.zeros((places, w.shape[1])), np.zeros((places, w.shape[1]))
    y = np.zeros_like(z)
    for e in range(w.shape[0]):
        at = slice(offsets[e], offsets[e + 1])
        z[at] = rows[at] @ w[e].T + (bias[e] if bias is not None else 0.0)
        size[at] = np.abs(rows[at]) @ np.abs(w[e]).T + (np.abs(bias[e]) if bias is not None else 0.0)
        y[at] = z[at] * slope(slope_at[at], activation) if slope_at is not None else act(z[at], activation)
    return y, z, size


def weight_gradient(dy, x, offsets, order=None, per_row=1):
    """(dw, db, sum of the absolute products of dw, of db)."""
    rows = rows_of(x, order, per_row, dy.shape[0])
    groups = len(offsets) - 1
    dw, db = np.zeros((groups, dy.shape[1], x.shape[1])), np.zeros((groups, dy.shape[1]))
    dw_size, db_size = np.zeros_like(dw), np.zeros_like(db)
    for e in range(groups):
        at = slice(offsets[e], offsets[e + 1])
        dw[e], db[e] = dy[at].T @ rows[at], dy[at].sum(0)
        dw_size[e], db_size[e] = np.abs(dy[at]).T @ np.abs(rows[at]), np.abs(dy[at]).sum(0)
    return dw, db, dw_size, db_size


def combine(values, slots, weights=None):
    y = np.zeros((slots.shape[0], values.shape[1]))
    for i in range(slots.shape[0]):
        for j in range(slots.shape[1]):
            if slots[i, j] >= 0:
                y[i] += (1.0 if weights is None else weights[i, j]) * values[slots[i, j]]
    return y


def combine_gradient(dy, values, slots, weights=None):
    dvalues, dweights = np.zeros(values.shape), np.zeros(slots.shape)
    for i in range(slots.shape[0]):
        for j in range(slots.shape[1]):
            if slots[i, j] >= 0:
                dvalues[slots[i, j]] += (1.0 if weights is None else weights[i, j]) * dy[i]
                dweights[i, j] = dy[i] @ values[slots[i, j]]
    return dvalues, dweights


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, decay, scale=1.0):
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p - lr * decay * p - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v


def decode_first(codes, scales):
    t = codes.astype(np.float64) / 127.0
    return t * np.abs(t) * np.repeat(scales.astype(np.float64), BLOCK)[:codes.size]


def decode_second(codes, scales):
    return (codes.astype(np.float64) / 255.0) ** 4 * np.repeat(scales.astype(np.float64), BLOCK)[:codes.size]


def _scaled(magnitude, most):
    """(scales of the blocks, every magnitude in units where its block's scale is `most`)."""
    scales = np.array([magnitude[b:b + BLOCK].max() for b in range(0, magnitude.size, BLOCK)])
    scales[scales < 2.0 ** -126] = 0.0
    each = np.repeat(scales, BLOCK)[:magnitude.size]
    return scales, np.where(each > 0, magnitude / np.where(each > 0, each, 1.0) * most, 0.0)


def _codes(t, power, most, u):
    """The nearest codes, or dithered ones: border between c and c + 1 at c^p + u ((c + 1)^p - c^p)."""
    if u is None:
        return np.floor(t ** (1.0 / power) + 0.5)
    c = np.floor(t ** (1.0 / power))
    return np.minimum(c + (t >= c ** power + u * ((c + 1.0) ** power - c ** power)), most)


def encode_first(m, u=None):
    """(codes, scales, t) with (c - 1/2)^2 <= t < (c + 1/2)^2, or dithered with u; codes carry the sign."""
    scales, t = _scaled(np.abs(m), 127.0 ** 2)
    return np.sign(m) * _codes(t, 2, 127, u), scales, t


def philox(counter, key):
    """Philox4x32 with 10 rounds (Salmon et al., SC'11): counter [.., 4] and key (two words) as unsigned 32-bit numbers."""
    c, (k0, k1), low = np.asarray(counter, dtype=np.uint64), (int(k) for k in key), np.uint64(0xFFFFFFFF)
    c = [c[..., i].copy() for i in range(4)]
    for r in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64((k0 + r * 0x9E3779B9) & 0xFFFFFFFF), p1 & low,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64((k1 + r * 0xBB67AE85) & 0xFFFFFFFF), p0 & low]
    return np.stack(c, -1)


def draws(n, step, second):
    """u of every element of a tensor: eight of 16 bits a call, the low half of a word first."""
    eighth = np.arange(-(-n // 8))
    counter = np.stack([eighth & 0xFFFFFFFF, eighth >> 32, np.full_like(eighth, int(second)), np.zeros_like(eighth)], -1)
    words = philox(counter, (step & 0xFFFFFFFF, step >> 32))
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(-1)
    return (halves[:n].astype(np.float64) + 0.5) / 65536.0


def encode_second(v, u=None):
    """(codes, scales, t), to the fourth power; a code is at least 1 where v > 0."""
    scales, t = _scaled(v, 255.0 ** 4)
    codes = _codes(t, 4, 255, u)
    return np.where(t > 0, np.maximum(codes, 1.0), 0.0), scales, t


# ---- routing by scores, dense products, the norm


def scores(logits, score):
    """s and its logarithm, -inf where there is no score."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -math.inf, x)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        if score == "sigmoid":
            s = 1.0 / (1.0 + np.exp(-x))
            log_s = np.where(x > -math.inf, np.minimum(x, 0.0) - np.log1p(np.exp(-np.abs(x))), -math.inf)
        else:
            top = x.max(1, keepdims=True)
            e = np.exp(x - np.where(np.isfinite(top), top, 0.0))
            total = e.sum(1, keepdims=True)
            s = e / total
            log_s = np.where(x > -math.inf, x - np.where(np.isfinite(top), top, 0.0) - np.log(total), -math.inf)
    return x, s, log_s


def route_scored(logits, k, score="sigmoid", bias=None, groups=1, top_groups=1, group_best=1, normalize=True, scale=1.0):
    """(experts, weights, offsets, order, slots): Python loops over rows, groups and slots."""
    x, s, log_s = scores(logits, score)
    n, n_experts = x.shape
    size = n_experts // groups
    experts, weights = np.full((n, k), -1, np.int32), np.zeros((n, k))
    for i in range(n):
        broken = score == "softmax" and not x[i].max() < math.inf
        by_logit = bias is None or broken
        c = x[i].copy() if by_logit else np.where(x[i] > -math.inf, s[i] + bias.astype(np.float64), -math.inf)
        c[np.isnan(c)] = -math.inf
        sums = c if not by_logit or group_best == 1 or broken else np.where(x[i] > -math.inf, s[i], -math.inf)
        ranking = []
        for g in range(groups):
            there = sorted((v for v in sums[g * size:(g + 1) * size] if v > -math.inf), reverse=True)[:group_best]
            if there:
                ranking.append((-sum(there), g))
        opened = [g for _, g in sorted(ranking)[:top_groups]]
        row = sorted((-c[e], e) for g in opened for e in range(g * size, (g + 1) * size) if c[e] > -math.inf)[:k]
        if not row:
            continue
        chosen = [e for _, e in row]
        if broken:
            share = np.full(len(chosen), math.nan)
        elif normalize:
            top = max(log_s[i, e] for e in chosen)
            share = np.exp(np.array([log_s[i, e] - top for e in chosen]))
            share /= share.sum()
        else:
            share = np.exp(log_s[i, chosen])
        experts[i, :len(chosen)] = chosen
        weights[i, :len(chosen)] = scale * share
    order, offsets = [], [0]
    flat = experts.reshape(-1)
    for e in range(n_experts):
        order.extend(np.flatnonzero(flat == e).tolist())
        offsets.append(len(order))
    slots = np.full(n * k, -1, np.int32)
    slots[order] = np.arange(len(order))
    return experts, weights, np.array(offsets, np.int32), np.array(order + [-1] * (n * k - len(order)), np.int32), slots.reshape(n, k)


def route_scored_gradient(logits, experts, weights, dweights, score="sigmoid", normalize=True, scale=1.0):
    """By the logarithms of the scores: d w_j = w_j (d log s_j [- sum w_i / scale d log s_i])."""
    x, s, _ = scores(logits, score)
    out = np.zeros(x.shape)
    for i in range(x.shape[0]):
        there = [j for j in range(experts.shape[1]) if experts[i, j] >= 0]
        inner = sum(weights[i, j] * dweights[i, j] for j in there) / scale if normalize else 0.0
        total = 0.0
        for j in there:
            back = weights[i, j] * (dweights[i, j] - inner)   # of log s_j
            out[i, experts[i, j]] += back / (1.0 + math.exp(min(x[i, experts[i, j]], 700.0))) if score == "sigmoid" else back
            total += back
        if score == "softmax" and there and not normalize:
            out[i] -= s[i] * total
    return out


def balance_bias(bias, offsets, rate):
    count = np.diff(np.asarray(offsets, dtype=np.int64))
    return np.asarray(bias, dtype=np.float64) + rate * np.sign(count.sum() - len(count) * count)


def dense(x, w, bias=None, activation=None, residual=None, slope_at=None):
    """(y, z, sum of the absolute products)."""
    z = x @ w.T + (0.0 if bias is None else bias)
    size = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    if slope_at is not None:
        return z * slope(slope_at, activation), z, size
    return act(z, activation) + (0.0 if residual is None else residual), z, size


def dense_gradient(dy, x, w, activation=None, z=None):
    """(dx, dw, db, dz)."""
    dz = dy * (slope(z, activation) if activation not in (None, "none") else 1.0)
    return dz @ w, dz.T @ x, dz.sum(0), dz


def gradient_norm(grads, max_norm=math.inf, grad_scale=1.0):
    """(norm, scale)."""
    norm = abs(grad_scale) * math.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    return norm, grad_scale if norm <= max_norm else grad_scale * (max_norm / norm)
