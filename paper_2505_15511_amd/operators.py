"""The operators of a learned map: routers, products grouped by expert and dense ones, weighted sum, AdamW, the gradients' norm (the second
half of include/nomad.h).

Tensors live on one GPU; a call checks them, takes what it returns from torch's allocator, enqueues the library's kernels on the
current stream (or `stream`) and returns without waiting.  Gradients are calls of their own: the framework has no
tape.  Tensors that do not fit each other raise ValueError, numbers that the library refuses NomadError, both before anything is
enqueued."""
from __future__ import annotations

import array
import ctypes as C
import itertools
import math
import operator
from typing import NamedTuple

import torch

from . import binding
from .binding import NomadError, load_library

MAX_K, MAX_EXPERTS, BLOCK = 8, 16384, 256
MAX_GROUPS = 64
SCORES = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_get_dtype = operator.attrgetter("dtype")


def _all_tensors(things):
    return all(issubclass(kind, torch.Tensor) for kind in set(map(type, things)))


def _dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _on(device, *tensors):
    """The tensors that are not None live on `device` (a torch.device of a GPU)."""
    if device.type != "cuda":
        raise ValueError("the operators take tensors on the GPU")
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"a tensor is on {t.device}, another one on {device}")


def _whole(t, name, dtype, shape):
    """`t` is contiguous, of that type and shape."""
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _rows(t, name, columns=None):
    """(rows, columns, stride) of a matrix whose columns are contiguous."""
    shape = t.shape
    if len(shape) != 2 or (columns is not None and shape[1] != columns):
        raise ValueError(f"{name} must be a matrix" + (f" of {columns} columns" if columns is not None else "") + f", got shape {tuple(shape)}")
    rows, columns = shape
    apart, beside = t.stride()
    if beside != 1 and columns > 1 and rows:
        raise ValueError(f"the columns of {name} must be contiguous (strides {t.stride()})")
    return rows, columns, apart if rows > 1 else columns


def _matrix(t, name):
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix, got shape {tuple(t.shape)}")
    return t.shape


def _stream(device, stream, used):
    """The stream of a call.  One other than the current stream waits (the host does not) for what the current one has been given so
    far: it may be making the inputs, or working on what a result's memory belonged to before; and what the call uses of
    torch's memory is not handed out again before that stream has come by here."""
    current = torch._C._cuda_getCurrentRawStream(device.index)   # the handle alone: a Stream object takes as long as a small copy
    if stream is None or int(stream) == current:
        return current
    other = torch.cuda.ExternalStream(int(stream), device=device)
    other.wait_stream(torch.cuda.current_stream(device))
    for t in used:
        if t is not None and t.numel():
            t.record_stream(other)
    return int(stream)


def _check(rc, name):
    if rc:
        raise NomadError(rc, name)


class Routing(NamedTuple):
    """What `route` returns (include/nomad.h): experts int32 [n, k], weights float32 [n, k], offsets int32 [n_experts + 1],
    order int32 [n k], slots int32 [n, k]."""
    experts: object
    weights: object
    offsets: object
    order: object
    slots: object


def route(logits, k, normalize=True, stream=None) -> Routing:
    """nomad_route: the k experts with the largest logits of every row [n, n_experts], their weights, and the rows in the order
    of their experts."""
    device = logits.device
    _on(device)
    code = _dtype(logits, "logits")
    n, experts, stride = _rows(logits, "logits")
    k = int(k)
    if not 1 <= k <= min(MAX_K, experts) or experts > MAX_EXPERTS:
        raise ValueError(f"k = {k} of {experts} experts: 1 <= k <= {MAX_K} and no more than there are (at most {MAX_EXPERTS})")
    lib = load_library()
    need = lib.nomad_route_workspace(n, experts, k)
    chosen, slots = torch.empty(n, k, dtype=torch.int32, device=device), torch.empty(n, k, dtype=torch.int32, device=device)
    weights, order = torch.empty(n, k, dtype=torch.float32, device=device), torch.empty(n * k, dtype=torch.int32, device=device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    st = _stream(device, stream, (logits, chosen, weights, offsets, order, slots, work))
    _check(lib.nomad_route(logits.data_ptr(), code, n, stride, experts, k, 1 if normalize else 0, chosen.data_ptr(), weights.data_ptr(), offsets.data_ptr(),
                           order.data_ptr(), slots.data_ptr(), work.data_ptr() if need else None, need, device.index, st or None), "nomad_route")
    out = Routing(chosen, weights, offsets, order, slots)
    return out


def route_gradient(logits, routing, dweights, normalize=True, stream=None):
    """nomad_route_gradient: the gradient of the logits from that of the weights; normalize as in the call of `route`."""
    device = logits.device
    _on(device, routing.experts, routing.weights, dweights)
    code = _dtype(logits, "logits")
    n, experts, stride = _rows(logits, "logits")
    _, k = _matrix(routing.experts, "routing.experts")
    _whole(routing.experts, "routing.experts", torch.int32, (n, k))
    _whole(routing.weights, "routing.weights", torch.float32, (n, k))
    _whole(dweights, "dweights", torch.float32, (n, k))
    out = torch.empty(n, experts, dtype=logits.dtype, device=device)
    st = _stream(device, stream, (logits, routing.experts, routing.weights, dweights, out))
    _check(load_library().nomad_route_gradient(logits.data_ptr(), code, n, stride, experts, k, 1 if normalize else 0, routing.experts.data_ptr(),
                                               routing.weights.data_ptr(), dweights.data_ptr(), out.data_ptr(), device.index, st or None), "nomad_route_gradient")
    return out


def _scoring(score, normalize, groups, top_groups, group_best, bias, scale):
    if not isinstance(score, str) or score not in SCORES:
        raise ValueError(f"score must be one of {sorted(SCORES)}")
    return binding.SCORING.pack(binding.SCORING.size, SCORES[score], 1 if normalize else 0, groups, top_groups, group_best, bias.data_ptr() if bias is not None else 0, scale)


def _scale(scale):
    scale = float(scale)
    if not math.isfinite(scale) or not 1e-37 < abs(scale) < 1e37:
        raise ValueError("scale must be a float32 number other than 0")
    return scale


def route_scored(logits, k, score="sigmoid", bias=None, groups=1, top_groups=1, group_best=1, normalize=True, scale=1.0, stream=None) -> Routing:
    """nomad_route_scored: the k experts of every row [n, n_experts] with the largest score ("sigmoid" or "softmax" of the logits) plus
    bias (None, or float32 [n_experts]: it has a say in the choice alone), in the top_groups of `groups` runs of neighbouring experts, by
    their group_best (1 or 2) largest; weights are scale times the scores, renormalised or not.  Returns what `route` returns."""
    device = logits.device
    _on(device, bias)
    code = _dtype(logits, "logits")
    n, experts, stride = _rows(logits, "logits")
    k, groups, top_groups, group_best = int(k), int(groups), int(top_groups), int(group_best)
    if not 1 <= k <= min(MAX_K, experts) or experts > MAX_EXPERTS:
        raise ValueError(f"k = {k} of {experts} experts: 1 <= k <= {MAX_K} and no more than there are (at most {MAX_EXPERTS})")
    if not 1 <= groups <= MAX_GROUPS or experts % groups:
        raise ValueError(f"{experts} experts are not cut into {groups} groups (at most {MAX_GROUPS})")
    if not 1 <= top_groups <= groups or group_best not in (1, 2) or k > top_groups * (experts // groups):
        raise ValueError(f"{top_groups} of {groups} groups by their {group_best} best: 1 <= top_groups <= groups, group_best 1 or 2, and room for k = {k}")
    if bias is not None:
        _whole(bias, "bias", torch.float32, (experts,))
    scoring = _scoring(score, normalize, groups, top_groups, group_best, bias, _scale(scale))
    lib = load_library()
    need = lib.nomad_route_workspace(n, experts, k)
    chosen, slots = torch.empty(n, k, dtype=torch.int32, device=device), torch.empty(n, k, dtype=torch.int32, device=device)
    weights, order = torch.empty(n, k, dtype=torch.float32, device=device), torch.empty(n * k, dtype=torch.int32, device=device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    st = _stream(device, stream, (logits, bias, chosen, weights, offsets, order, slots, work))
    _check(lib.nomad_route_scored(logits.data_ptr(), code, n, stride, experts, k, scoring, chosen.data_ptr(), weights.data_ptr(), offsets.data_ptr(), order.data_ptr(),
                                  slots.data_ptr(), work.data_ptr() if need else None, need, device.index, st or None), "nomad_route_scored")
    return Routing(chosen, weights, offsets, order, slots)


def route_scored_gradient(logits, routing, dweights, score="sigmoid", normalize=True, scale=1.0, stream=None):
    """nomad_route_scored_gradient: the gradient of the logits from that of the weights; score, normalize and scale as in the call of
    `route_scored`.  The bias has none (`balance_bias` is its step)."""
    device = logits.device
    _on(device, routing.experts, routing.weights, dweights)
    code = _dtype(logits, "logits")
    n, experts, stride = _rows(logits, "logits")
    _, k = _matrix(routing.experts, "routing.experts")
    _whole(routing.experts, "routing.experts", torch.int32, (n, k))
    _whole(routing.weights, "routing.weights", torch.float32, (n, k))
    _whole(dweights, "dweights", torch.float32, (n, k))
    scoring = _scoring(score, normalize, 1, 1, 1, None, _scale(scale))
    out = torch.empty(n, experts, dtype=logits.dtype, device=device)
    st = _stream(device, stream, (logits, routing.experts, routing.weights, dweights, out))
    _check(load_library().nomad_route_scored_gradient(logits.data_ptr(), code, n, stride, experts, k, scoring, routing.experts.data_ptr(), routing.weights.data_ptr(),
                                                      dweights.data_ptr(), out.data_ptr(), device.index, st or None), "nomad_route_scored_gradient")
    return out


def balance_bias(bias, offsets, rate, stream=None):
    """nomad_balance_bias: bias [n_experts], float32, with `rate` more for experts that have fewer rows than the mean (offsets of a
    routing), and less for those that have more; a new tensor."""
    device = bias.device
    _on(device, offsets)
    if bias.dim() != 1 or not 1 <= bias.shape[0] <= MAX_EXPERTS:
        raise ValueError(f"bias must be a tensor of 1 to {MAX_EXPERTS} experts, got shape {tuple(bias.shape)}")
    experts = bias.shape[0]
    _whole(bias, "bias", torch.float32, (experts,))
    _whole(offsets, "offsets", torch.int32, (experts + 1,))
    if not abs(rate) <= torch.finfo(torch.float32).max:
        raise ValueError("rate must be a float32 number")
    out = torch.empty_like(bias)
    st = _stream(device, stream, (bias, offsets, out))
    _check(load_library().nomad_balance_bias(bias.data_ptr(), offsets.data_ptr(), experts, float(rate), out.data_ptr(), device.index, st or None), "nomad_balance_bias")
    return out


def _grouping(x_rows, offsets, order, per_row, rows):
    """Checks of what says which row of x stands at which place; the number of places."""
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or not offsets.is_contiguous() or offsets.shape[0] < 2:
        raise ValueError("offsets must be a contiguous int32 tensor of one entry more than there are groups")
    places = x_rows
    if order is not None:
        if order.dtype != torch.int32 or order.dim() != 1 or not order.is_contiguous():
            raise ValueError("order must be a contiguous int32 tensor")
        if not 1 <= int(per_row) < 2 ** 31:
            raise ValueError("per_row must be at least 1, and 32 bits")
        places = order.shape[0]
        if places and not x_rows:
            raise ValueError("order asks for rows of an empty x")
    if rows is not None and rows != places:
        raise ValueError(f"{places} places, but {rows} rows")
    return places


def grouped_product(x, w, offsets, bias=None, activation=None, order=None, per_row=1, keep=False, slope_at=None, out_dtype=None, stream=None):
    """nomad_grouped_product: y_p = act(x_p W_e^T + b_e) for the places p of every group e (offsets [E + 1]), x_p = x[p] or
    x[order[p] // per_row].  w [E, out, in] in either order of its last two strides; keep=True returns (y, z) with z the products
    before the activation; slope_at=z multiplies by the activation's slope at z instead (the way back)."""
    device = x.device
    _on(device, w, offsets, bias, order, slope_at)
    code = _dtype(x, "x")
    if not isinstance(activation, (str, type(None))) or activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(k for k in ACTIVATIONS if k)}")
    x_rows, columns, x_stride = _rows(x, "x")
    shape = w.shape
    if len(shape) != 3 or w.dtype != x.dtype or shape[2] != columns or 0 in shape:
        raise ValueError(f"w must be [experts, out, {columns}] of {x.dtype}, got {tuple(shape)} of {w.dtype}")
    groups, out, inner = shape
    places = _grouping(x_rows, offsets, order, per_row, None)
    if offsets.shape[0] != groups + 1:
        raise ValueError(f"{groups} groups need {groups + 1} offsets, got {offsets.shape[0]}")
    sg, so, si = w.stride()
    if inner == 1:
        si = 1
    if out == 1 and si != 1:
        so = 1
    if si != 1 and so != 1:
        raise ValueError(f"one of the last two strides of w must be 1 (strides {w.stride()}): .contiguous() copies it")
    if bias is not None:
        if bias.dtype != x.dtype or tuple(bias.shape) != (groups, out) or (out > 1 and bias.stride(1) != 1):
            raise ValueError(f"bias must be [{groups}, {out}] of {x.dtype} with contiguous rows")
    z_stride = 0
    if slope_at is not None:
        if bias is not None or keep:
            raise ValueError("slope_at goes without bias and keep")
        if slope_at.dtype != x.dtype or _matrix(slope_at, "slope_at")[0] != places:
            raise ValueError(f"slope_at must be [{places}, {out}] of {x.dtype}")
        _, _, z_stride = _rows(slope_at, "slope_at", out)
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's type or float32")
    y = torch.empty(places, out, dtype=out_dtype, device=device)
    z = torch.empty(places, out, dtype=x.dtype, device=device) if keep else None
    st = _stream(device, stream, (x, w, offsets, bias, order, slope_at, y, z))
    a = binding.GROUPED_PRODUCT_ARGS.pack(
        binding.GROUPED_PRODUCT_ARGS.size, code, _DTYPES[out_dtype], ACTIVATIONS[activation], groups, int(per_row) if order is not None else 1, inner, out, places, x_rows,
        offsets.data_ptr(), order.data_ptr() if order is not None else 0, x.data_ptr(), x_stride, w.data_ptr(), sg if groups > 1 else 0, so, si,
        bias.data_ptr() if bias is not None else 0, bias.stride(0) if bias is not None and groups > 1 else 0,
        slope_at.data_ptr() if slope_at is not None else 0, z_stride, y.data_ptr(), out, z.data_ptr() if keep else 0, out, st, device.index)
    _check(load_library().nomad_grouped_product(a), "nomad_grouped_product")
    return (y, z) if keep else y


def grouped_weight_gradient(dy, x, offsets, order=None, per_row=1, bias=True, out_dtype=None, stream=None):
    """nomad_grouped_weight_gradient: (dW [E, out, in], db [E, out] float32 or None) from dy [places, out] and the x, offsets and
    order of the product."""
    device = x.device
    _on(device, dy, offsets, order)
    code = _dtype(x, "x")
    if dy.dtype != x.dtype:
        raise ValueError(f"dy is {dy.dtype}, x {x.dtype}")
    x_rows, inner, x_stride = _rows(x, "x")
    rows, out, dy_stride = _rows(dy, "dy")
    _grouping(x_rows, offsets, order, per_row, rows)
    groups = offsets.shape[0] - 1
    if inner < 1 or out < 1:
        raise ValueError("x and dy need columns")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's type or float32")
    lib = load_library()
    dw = torch.empty(groups, out, inner, dtype=out_dtype, device=device)
    db = torch.empty(groups, out, dtype=torch.float32, device=device) if bias else None
    need = lib.nomad_grouped_gradient_workspace(rows, groups, inner, out, code)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    st = _stream(device, stream, (x, dy, offsets, order, dw, db, work))
    a = binding.GROUPED_GRADIENT_ARGS.pack(
        binding.GROUPED_GRADIENT_ARGS.size, code, _DTYPES[out_dtype], groups, int(per_row) if order is not None else 1, inner, out, rows, x_rows, offsets.data_ptr(),
        order.data_ptr() if order is not None else 0, dy.data_ptr(), dy_stride, x.data_ptr(), x_stride, dw.data_ptr(), db.data_ptr() if bias else 0,
        work.data_ptr() if need else 0, need, st, device.index)
    _check(lib.nomad_grouped_weight_gradient(a), "nomad_grouped_weight_gradient")
    return dw, db


def _weights(w, dtype, columns):
    """(out, in, strides) of a weight matrix in either order."""
    shape = w.shape
    if len(shape) != 2 or w.dtype != dtype or (columns is not None and shape[1] != columns) or 0 in shape:
        raise ValueError(f"w must be [out, {'in' if columns is None else columns}] of {dtype}, got {tuple(shape)} of {w.dtype}")
    out, inner = shape
    so, si = w.stride()
    if inner == 1:
        si = 1
    if out == 1 and si != 1:
        so = 1
    if si != 1 and so != 1:
        raise ValueError(f"one of the strides of w must be 1 (strides {w.stride()}): .contiguous() copies it")
    return out, inner, so, si


def _activation(activation):
    if not isinstance(activation, (str, type(None))) or activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(k for k in ACTIVATIONS if k)}")
    return ACTIVATIONS[activation]


def dense_product(x, w, bias=None, activation=None, residual=None, keep=False, slope_at=None, out_dtype=None, stream=None):
    """nomad_dense_product: y = act(x w^T + bias) + residual, x [n, in], w [out, in] in either order of its strides, bias [out],
    residual [n, out]; keep=True returns (y, z) with z the products before the activation; slope_at=z multiplies by the activation's slope at z
    instead (the way back)."""
    device = x.device
    _on(device, w, bias, residual, slope_at)
    code, act = _dtype(x, "x"), _activation(activation)
    n, columns, x_stride = _rows(x, "x")
    out, inner, so, si = _weights(w, x.dtype, columns)
    if bias is not None:
        _whole(bias, "bias", x.dtype, (out,))
    if slope_at is not None and (bias is not None or residual is not None or keep):
        raise ValueError("slope_at goes without bias, residual and keep")
    strides = [0, 0]
    for i, (t, name) in enumerate(((residual, "residual"), (slope_at, "slope_at"))):
        if t is not None:
            if t.dtype != x.dtype or _matrix(t, name)[0] != n:
                raise ValueError(f"{name} must be [{n}, {out}] of {x.dtype}")
            strides[i] = _rows(t, name, out)[2]
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's type or float32")
    lib = load_library()
    y = torch.empty(n, out, dtype=out_dtype, device=device)
    z = torch.empty(n, out, dtype=x.dtype, device=device) if keep else None
    need = lib.nomad_dense_workspace(n, inner, out, code)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    st = _stream(device, stream, (x, w, bias, residual, slope_at, y, z, work))
    a = binding.DENSE_ARGS.pack(
        binding.DENSE_ARGS.size, code, _DTYPES[out_dtype], act, inner, out, n, x.data_ptr(), x_stride, w.data_ptr(), so, si, bias.data_ptr() if bias is not None else 0,
        residual.data_ptr() if residual is not None else 0, strides[0], slope_at.data_ptr() if slope_at is not None else 0, strides[1], y.data_ptr(), out,
        z.data_ptr() if keep else 0, out, work.data_ptr() if need else 0, need, st, device.index)
    _check(lib.nomad_dense_product(a), "nomad_dense_product")
    return (y, z) if keep else y


def dense_gradient(dy, x, w, activation=None, z=None, need_dx=True, need_dw=True, bias=True, out_dtype=None, stream=None):
    """nomad_dense_gradient: (dx [n, in], dW [out, in] of out_dtype, db [out] float32) of `dense_product` from dy [n, out]; with an
    activation z is what keep=True returned.  What is not needed is None (db comes with dW); the residual's gradient is dy."""
    device = x.device
    _on(device, dy, w, z)
    code, act = _dtype(x, "x"), _activation(activation)
    n, columns, x_stride = _rows(x, "x")
    out, inner, so, si = _weights(w, x.dtype, columns)
    if dy.dtype != x.dtype or _matrix(dy, "dy")[0] != n:
        raise ValueError(f"dy must be [{n}, {out}] of {x.dtype}")
    dy_stride, z_stride = _rows(dy, "dy", out)[2], 0
    if act:
        if z is None or z.dtype != x.dtype or _matrix(z, "z")[0] != n:
            raise ValueError(f"with an activation z must be [{n}, {out}] of {x.dtype}")
        z_stride = _rows(z, "z", out)[2]
    if not need_dx and not need_dw:
        raise ValueError("neither gradient is asked for")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's type or float32")
    lib = load_library()
    dx = torch.empty(n, inner, dtype=x.dtype, device=device) if need_dx else None
    dw = torch.empty(out, inner, dtype=out_dtype, device=device) if need_dw else None
    db = torch.empty(out, dtype=torch.float32, device=device) if need_dw and bias else None
    need = lib.nomad_dense_gradient_workspace(n, inner, out, code, act)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    st = _stream(device, stream, (dy, x, w, z if act else None, dx, dw, db, work))
    pointer = lambda t: t.data_ptr() if t is not None else 0   # noqa: E731
    a = binding.DENSE_GRADIENT_ARGS.pack(
        binding.DENSE_GRADIENT_ARGS.size, code, _DTYPES[out_dtype], act, inner, out, n, dy.data_ptr(), dy_stride, z.data_ptr() if act else 0, z_stride, x.data_ptr(), x_stride,
        w.data_ptr(), so, si, pointer(dx), inner, pointer(dw), pointer(db), pointer(work), need, st, device.index)
    _check(lib.nomad_dense_gradient(a), "nomad_dense_gradient")
    return dx, dw, db


def combine(values, slots, weights=None, stream=None):
    """nomad_combine: y_i = sum_j weights[i, j] values[slots[i, j]] (weights None: ones)."""
    device = values.device
    _on(device, slots, weights)
    code = _dtype(values, "values")
    n_values, d, stride = _rows(values, "values")
    n, k = _matrix(slots, "slots")
    _whole(slots, "slots", torch.int32, (n, k))
    if weights is not None:
        _whole(weights, "weights", torch.float32, (n, k))
    y = torch.empty(n, d, dtype=values.dtype, device=device)
    st = _stream(device, stream, (values, slots, weights, y))
    _check(load_library().nomad_combine(values.data_ptr(), code, n_values, stride, d, slots.data_ptr(),
                                        weights.data_ptr() if weights is not None else None, n, k, y.data_ptr(), device.index, st or None), "nomad_combine")
    return y


def combine_gradient(dy, values, slots, weights=None, order=None, need_dvalues=True, need_dweights=True, stream=None):
    """nomad_combine_gradient: (dvalues like values, dweights [n, k] float32); what is not needed is None.  With `order` (of
    `route`) the places that no slot takes get zeros; without it every place must be some slot's."""
    device = values.device
    _on(device, dy, slots, weights, order)
    code = _dtype(values, "values")
    n_values, d, stride = _rows(values, "values")
    n, k = _matrix(slots, "slots")
    _whole(slots, "slots", torch.int32, (n, k))
    if weights is not None:
        _whole(weights, "weights", torch.float32, (n, k))
    if order is not None:
        _whole(order, "order", torch.int32, (n * k,))
        if n_values != n * k:
            raise ValueError(f"order says {n * k} places, values has {n_values}")
    if dy.dtype != values.dtype or _matrix(dy, "dy")[0] != n:
        raise ValueError(f"dy must be [{n}, {d}] of {values.dtype}")
    _, _, dy_stride = _rows(dy, "dy", d)
    if not need_dvalues and not need_dweights:
        raise ValueError("neither gradient is asked for")
    dvalues = torch.empty(n_values, d, dtype=values.dtype, device=device) if need_dvalues else None
    dweights = torch.empty(n, k, dtype=torch.float32, device=device) if need_dweights else None
    st = _stream(device, stream, (dy, values, slots, weights, order, dvalues, dweights))
    _check(load_library().nomad_combine_gradient(
        dy.data_ptr(), code, dy_stride, values.data_ptr(), n_values, stride, d, slots.data_ptr(), order.data_ptr() if order is not None else None,
        weights.data_ptr() if weights is not None else None, n, k, dvalues.data_ptr() if need_dvalues else None,
        dweights.data_ptr() if need_dweights else None, device.index, st or None), "nomad_combine_gradient")
    return dvalues, dweights


def gradient_norm(grads, max_norm=math.inf, grad_scale=None, stream=None):
    """nomad_gradient_norm: (norm, scale), float32 tensors of one element on the GPU: the norm of all tensors together, and the factor that brings it
    to max_norm at most, as `adamw_step` takes it (grad_scale).  An infinite gradient makes
    the factor 0, and is NaN in the step. A tensor that is in the list twice counts twice.  grad_scale: None, or a factor that the gradients have yet to be multiplied
    by, which norm and scale then contain."""
    grads = list(grads)
    if not grads:
        raise ValueError("there are no gradients")
    if not _all_tensors(grads):
        raise ValueError("gradients must be tensors")
    device = grads[0].device
    _on(device, grad_scale)
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
        raise ValueError("grad_scale must be one float32 element")
    max_norm = float(max_norm)
    if not max_norm >= 0.0:
        raise ValueError("max_norm must not be negative")
    if set(map(torch.Tensor.get_device, grads)) != {device.index} or not all(map(torch.Tensor.is_contiguous, grads)):
        raise ValueError(f"gradients must be contiguous and on {device}")
    dtypes = set(map(_get_dtype, grads))
    if not dtypes <= _DTYPES.keys():
        raise ValueError("gradients must be float32, bfloat16 or float16")
    lib, count = load_library(), len(grads)
    # the structures' fields, each a slice (120 tensors: a third of the time of taking them one by one)
    words = [_DTYPES[next(iter(dtypes))]] * (3 * count)
    words[::3], words[1::3] = list(map(torch.Tensor.data_ptr, grads)), list(map(torch.Tensor.numel, grads))
    if len(dtypes) > 1:
        words[2::3] = [_DTYPES[g.dtype] for g in grads]
    flat = array.array("q", words)
    out = torch.empty(2, dtype=torch.float32, device=device)
    need = lib.nomad_gradient_norm_workspace(count)
    work = torch.empty(need, dtype=torch.uint8, device=device)
    st = _stream(device, stream, grads + [grad_scale, out, work])
    at = out.data_ptr()
    _check(lib.nomad_gradient_norm(flat.buffer_info()[0], count, max_norm, grad_scale.data_ptr() if grad_scale is not None else None, at, at + 4, work.data_ptr(), need,
                                   device.index, st or None), "nomad_gradient_norm")
    return out[:1], out[1:]


class State8(NamedTuple):
    """An average in 8 bits: codes (int8 of the first, uint8 of the second) [n] and the scales float32 of blocks of 256."""
    codes: object
    scales: object


def adamw_state(param, bits=32):
    """(first, second) averages of a tensor before its first step: float32 tensors, or State8 with bits=8."""
    if bits == 32:
        return torch.zeros(param.shape, dtype=torch.float32, device=param.device), torch.zeros(param.shape, dtype=torch.float32, device=param.device)
    if bits != 8:
        raise ValueError("bits must be 8 or 32")
    n = param.numel()
    blocks = -(-n // BLOCK)
    return tuple(State8(torch.zeros(n, dtype=d, device=param.device), torch.zeros(blocks, dtype=torch.float32, device=param.device)) for d in (torch.int8, torch.uint8))


def adamw_step(params, grads, first, second, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None, dither=False, stream=None):
    """nomad_adamw_step: one step, in place, over all of the tensors at once.  first and second: the averages of `adamw_state`
    (all in 32 bits, or all in 8); step counts from 1; grad_scale: None or a float32 tensor of one element on the GPU.  dither, for
    averages in 8 bits: codes that are right on average instead of the nearest, which a beta2 above 0.99 needs to forget."""
    params, grads, first, second = list(params), list(grads), list(first), list(second)
    if not len(params) == len(grads) == len(first) == len(second):
        raise ValueError("params, grads, first and second must be lists of the same length")
    if not params:
        return
    eight = not isinstance(first[0], torch.Tensor)
    device = params[0].device
    if dither and not eight:
        raise ValueError("dither is for averages in 8 bits")
    _on(device, grad_scale)
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
        raise ValueError("grad_scale must be one float32 element")
    # every check is a pass over all tensors by one C function: a step over a hundred small tensors takes the host longer than the GPU
    tensors = params + grads
    if eight:
        if any(isinstance(s, torch.Tensor) for s in itertools.chain(first, second)):
            raise ValueError("the states must all be in 32 bits, or all in 8")
        m, m_scale = [s[0] for s in first], [s[1] for s in first]
        v, v_scale = [s[0] for s in second], [s[1] for s in second]
        tensors += m + v + m_scale + v_scale
        wanted = ((m, {torch.int8}), (v, {torch.uint8}), (m_scale, {torch.float32}), (v_scale, {torch.float32}))
    else:
        if not (_all_tensors(first) and _all_tensors(second)):
            raise ValueError("the states must all be in 32 bits, or all in 8")
        m, v = first, second
        tensors += m + v
        wanted = ((m, {torch.float32}), (v, {torch.float32}))
    if set(map(torch.Tensor.get_device, tensors)) != {device.index} or not all(map(torch.Tensor.is_contiguous, tensors)):
        raise ValueError(f"tensors must be contiguous and on {device}")
    for which, dtypes in wanted:
        if set(map(_get_dtype, which)) != dtypes:
            raise ValueError("states are float32 in 32 bits; int8 and uint8 codes with float32 scales in 8")
    sizes = list(map(torch.Tensor.numel, params))
    if any(list(map(torch.Tensor.numel, which)) != sizes for which in (grads, m, v)):
        raise ValueError("a tensor, its gradient and its states must have as many elements")
    if eight:
        blocks = [-(-n // BLOCK) for n in sizes]
        if any(list(map(torch.Tensor.numel, which)) != blocks for which in (m_scale, v_scale)):
            raise ValueError(f"8-bit states have a scale for every {BLOCK} elements")
    codes = _DTYPES
    kinds = list(zip(map(_get_dtype, params), map(_get_dtype, grads)))
    for p, g in set(kinds):
        if p not in codes or g not in codes or (g != p and torch.float32 not in (p, g)):
            raise ValueError(f"no step for {p} with gradients in {g}")
    count, pointer = len(params), torch.Tensor.data_ptr
    none = [0] * count
    words = {k: codes[k[0]] | codes[k[1]] << 32 for k in set(kinds)}   # (p_dtype and g_dtype, two 32-bit fields)
    rows = zip(map(pointer, params), map(pointer, grads), map(pointer, m), map(pointer, v), map(pointer, m_scale) if eight else none,
               map(pointer, v_scale) if eight else none, sizes, map(words.__getitem__, kinds))
    flat = array.array("q", itertools.chain.from_iterable(rows))
    st = _stream(device, stream, tensors + [grad_scale])
    options = binding.ADAMW_OPTIONS.pack(binding.ADAMW_OPTIONS.size, 8 if eight else 32, int(step), float(lr), float(betas[0]), float(betas[1]), float(eps),
                                         float(weight_decay), grad_scale.data_ptr() if grad_scale is not None else 0, st, device.index, 1 if dither else 0)
    _check(load_library().nomad_adamw_step(flat.buffer_info()[0], count, options), "nomad_adamw_step")


def adamw_state_values(states, stream=None):
    """nomad_adamw_state_values: 8-bit averages (a list of State8, all first or all second ones) as float32 tensors."""
    states = [State8(*s) for s in states]
    if not states:
        return []
    device, dtype = states[0].codes.device, states[0].codes.dtype
    _on(device)
    if dtype not in (torch.int8, torch.uint8):
        raise ValueError("codes are int8 (first averages) or uint8 (second)")
    for s in states:
        n = s.codes.numel()
        _on(device, s.codes, s.scales)
        if s.codes.dtype != dtype or not s.codes.is_contiguous():
            raise ValueError("codes must be contiguous, and all first or all second averages")
        _whole(s.scales, "scales", torch.float32, (-(-n // BLOCK),))
    sizes = [s.codes.numel() for s in states]
    # one allocation; every tensor begins on a border of 16 bytes
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += -(-n // 4) * 4
    held = torch.empty(total, dtype=torch.float32, device=device)
    out = [held[at:at + n] for at, n in zip(starts, sizes)]
    count = len(states)
    addresses, words = C.c_void_p * count, C.c_int64 * count
    st = _stream(device, stream, [held] + [t for s in states for t in s])
    _check(load_library().nomad_adamw_state_values(addresses(*[s.codes.data_ptr() for s in states]), addresses(*[s.scales.data_ptr() for s in states]),
                                                   addresses(*[t.data_ptr() for t in out]), words(*sizes), count, 1 if dtype == torch.uint8 else 0, device.index,
                                                   st or None), "nomad_adamw_state_values")
    return out
