"""Binding of the experts' rows: the order of the places that a router chose, the
products grouped by expert, and the weighted sum of the experts' outputs.

The functions carry the C names (include/lapsum.h has their definitions) and only
check and marshal their arguments; the differentiable forms are
autograd.expert_matmul and autograd.expert_combine.

    w, idx = lapsum_route_forward(logits, 2)
    order, place, offsets = lapsum_expert_order(idx, experts)
    h = lapsum_expert_matmul(x, up, offsets, order=order, top_k=2)
    y = lapsum_expert_combine(lapsum_expert_matmul(torch.relu(h), down, offsets), place, w)
"""
from __future__ import annotations

import ctypes

from . import _check, _on_device, _ptr, _stream, _torch, _workspace, load
from .selection import _count, _device_tensor, _dtype, _expect, _node

__all__ = [
    "lapsum_expert_order_workspace_size", "lapsum_expert_order", "lapsum_expert_matmul",
    "lapsum_expert_matmul_weights_workspace_size", "lapsum_expert_matmul_weights",
    "lapsum_expert_combine", "lapsum_expert_combine_backward",
]

_lib = None


def _load():
    """The library with the signatures of this module declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = load()
    vp, i64, sz, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    lib.lapsum_expert_order_workspace_size.argtypes = [i64, i64]
    lib.lapsum_expert_order_workspace_size.restype = sz
    lib.lapsum_expert_order.argtypes = [vp, i64, i64, vp, vp, vp, vp, sz, vp]
    lib.lapsum_expert_order.restype = i32
    lib.lapsum_expert_matmul.argtypes = [vp, i32, i64, i64, vp, i64, vp, i64, i64, i64, i64, vp, vp, vp,
                                         i32, vp]
    lib.lapsum_expert_matmul.restype = i32
    lib.lapsum_expert_matmul_weights_workspace_size.argtypes = [i64, i64, i64, i64]
    lib.lapsum_expert_matmul_weights_workspace_size.restype = sz
    lib.lapsum_expert_matmul_weights.argtypes = [vp, i32, i64, i64, vp, i64, vp, i64, i64, i64, i64, vp,
                                                 i64, vp, vp, vp, sz, vp]
    lib.lapsum_expert_matmul_weights.restype = i32
    lib.lapsum_expert_combine.argtypes = [vp, i32, i64, i64, vp, vp, i64, i64, vp, i32, vp]
    lib.lapsum_expert_combine.restype = i32
    lib.lapsum_expert_combine_backward.argtypes = [vp, vp, i32, i64, i64, vp, vp, vp, i64, i64, i64, vp,
                                                   vp, vp]
    lib.lapsum_expert_combine_backward.restype = i32
    _lib = lib
    return lib


def _matrix_rows(x, name):
    """x as rows of its last dimension that are evenly apart: (tensor, stride)."""
    if x.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    if (x.stride(1) != 1 and x.shape[1] > 1) or (x.stride(0) < x.shape[1] and x.shape[0] > 1):
        x = x.contiguous()
    return x, (x.stride(0) if x.shape[0] > 1 else x.shape[1])


def _matrices(w, device, dtype):
    """w [experts, in, out] with one of the last two dimensions dense, and its strides."""
    _device_tensor(w, "weight", dtype)
    if w.dim() != 3 or w.device != device:
        raise ValueError(f"weight must be [experts, in, out] on {device}")
    se, si, so = w.stride()
    _, n_in, n_out = w.shape
    if not ((so == 1 and si >= n_out) or (si == 1 and so >= n_in)):
        w = w.contiguous()
        se, si, so = w.stride()
    return w, (ctypes.c_int64 * 3)(se, si, so)


def _offsets(offsets, experts, device):
    return _expect(offsets, "offsets", (experts + 1,), _torch().int32, device)


# ---------------------------------------------------------------- order ----
def lapsum_expert_order_workspace_size(count: int, experts: int) -> int:
    return int(_load().lapsum_expert_order_workspace_size(count, experts))


def lapsum_expert_order(indices, experts: int, *, workspace=None):
    """The places of indices, int32 of any shape, by expert: (order, place, offsets),
    int32 [places], the shape of indices, and [experts + 1].  order lists the places
    of expert 0, then 1 and so on, those of an index outside [0, experts) last; place
    is each place's position in it (-1 without an expert); expert e has positions
    offsets[e] to offsets[e + 1]."""
    node = _node()
    if node and workspace is None:
        try:
            out = node.expert_order(indices, experts)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(indices, "indices", torch.int32)
    at = indices.contiguous()
    experts = _count(experts, "experts")
    dev = at.device
    order = torch.empty(at.numel(), dtype=torch.int32, device=dev)
    place = torch.empty(at.shape, dtype=torch.int32, device=dev)
    offsets = torch.empty(max(experts, 0) + 1, dtype=torch.int32, device=dev)
    ws, nbytes = _workspace(lib.lapsum_expert_order_workspace_size(at.numel(), experts), dev, workspace)
    with _on_device(dev):
        _check(lib.lapsum_expert_order(_ptr(at), at.numel(), experts, _ptr(order), _ptr(place),
                                       _ptr(offsets), _ptr(ws), nbytes, _stream(dev)),
               "lapsum_expert_order")
    return order, place, offsets


# ------------------------------------------------------------- products ----
def lapsum_expert_matmul(x, weight, offsets, *, order=None, top_k: int = 1, dtype=None):
    """y[i] = x[row(i)] @ weight[e] for the rows i of each expert e, and zeros for the
    rows of none: [rows, out] of x's type, or float32 with dtype=torch.float32.
    x [x_rows, in] and weight [experts, in, out] (stored either way round) of one
    type; offsets int32 [experts + 1].  With order (int32 [rows], of
    lapsum_expert_order over [x_rows, top_k] places) row(i) = order[i] // top_k,
    else i."""
    node = _node()
    if node and dtype is None:
        try:
            out = node.expert_matmul(x, weight, offsets, order, top_k)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(x, "x")
    code = _dtype(x, "x")
    x, stride = _matrix_rows(x, "x")
    dev = x.device
    w, strides = _matrices(weight, dev, x.dtype)
    experts, n_in, n_out = w.shape
    if x.shape[1] != n_in:
        raise ValueError("x and weight must agree on `in`")
    _offsets(offsets, experts, dev)
    top_k = _count(top_k, "top_k")
    rows = x.shape[0]
    if order is not None:
        _expect(order, "order", (order.numel(),), torch.int32, dev)
        rows = order.numel()
    if dtype not in (None, x.dtype, torch.float32):
        raise ValueError("dtype must be that of x or float32")
    y = torch.empty((rows, n_out), dtype=dtype or x.dtype, device=dev)
    with _on_device(dev):
        _check(lib.lapsum_expert_matmul(_ptr(x), code, x.shape[0], stride, _ptr(order), top_k,
                                        _ptr(offsets), experts, rows, n_in, n_out, _ptr(w), strides,
                                        _ptr(y), _dtype(y, "y"), _stream(dev)), "lapsum_expert_matmul")
    return y


def lapsum_expert_matmul_weights_workspace_size(experts: int, rows: int, n_in: int, n_out: int) -> int:
    return int(_load().lapsum_expert_matmul_weights_workspace_size(experts, rows, n_in, n_out))


def lapsum_expert_matmul_weights(x, grad_y, offsets, like, *, order=None, top_k: int = 1, workspace=None):
    """The gradient of lapsum_expert_matmul with respect to its weight, in the
    shape, type and storage of `like` (the weight; strides only are read of it)."""
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(x, "x")
    code = _dtype(x, "x")
    x, stride = _matrix_rows(x, "x")
    dev = x.device
    _device_tensor(grad_y, "grad_y", x.dtype)
    g, g_stride = _matrix_rows(grad_y, "grad_y")
    experts, n_in, n_out = like.shape
    _offsets(offsets, experts, dev)
    rows = x.shape[0]
    if order is not None:
        _expect(order, "order", (order.numel(),), torch.int32, dev)
        rows = order.numel()
    if x.shape[1] != n_in or g.shape != (rows, n_out) or g.device != dev:
        raise ValueError("x, grad_y and the weight must agree on rows, `in` and `out`")
    if like.stride(1) == 1 and like.stride(2) != 1:
        grad = torch.empty((experts, n_out, n_in), dtype=x.dtype, device=dev).transpose(1, 2)
    else:
        grad = torch.empty((experts, n_in, n_out), dtype=x.dtype, device=dev)
    ws, nbytes = _workspace(lib.lapsum_expert_matmul_weights_workspace_size(experts, rows, n_in, n_out),
                            dev, workspace)
    with _on_device(dev):
        _check(lib.lapsum_expert_matmul_weights(
            _ptr(x), code, x.shape[0], stride, _ptr(order), _count(top_k, "top_k"), _ptr(offsets),
            experts, rows, n_in, n_out, _ptr(g), g_stride, _ptr(grad),
            (ctypes.c_int64 * 3)(*grad.stride()), _ptr(ws), nbytes, _stream(dev)),
               "lapsum_expert_matmul_weights")
    return grad


# ----------------------------------------------------------------- sums ----
def _places(place, device):
    torch = _torch()
    _device_tensor(place, "place", torch.int32)
    if place.dim() != 2 or not place.is_contiguous() or place.device != device:
        raise ValueError(f"place must be contiguous [tokens, top_k] on {device}")
    return place


def lapsum_expert_combine(y, place, weights=None, *, dtype=None):
    """out[t] = sum_j weights[t, j] y[place[t, j]]: y [rows, dim], place int32
    and weights float32 [tokens, top_k] (None: 1 each); [tokens, dim] of y's type
    (of any with a float32 y)."""
    node = _node()
    if node and dtype is None:
        try:
            out = node.expert_combine(y, place, weights)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(y, "y")
    code = _dtype(y, "y")
    if y.dim() != 2:
        raise ValueError("y must be [rows, dim]")
    y = y.contiguous()
    dev = y.device
    _places(place, dev)
    if weights is not None:
        _expect(weights, "weights", place.shape, torch.float32, dev)
    out = torch.empty((place.shape[0], y.shape[1]), dtype=dtype or y.dtype, device=dev)
    with _on_device(dev):
        _check(lib.lapsum_expert_combine(_ptr(y), code, y.shape[0], y.shape[1], _ptr(weights),
                                         _ptr(place), place.shape[0], place.shape[1], _ptr(out),
                                         _dtype(out, "out"), _stream(dev)), "lapsum_expert_combine")
    return out


def lapsum_expert_combine_backward(grad_out, y, place, weights, offsets):
    """(grad_y, grad_weights) of lapsum_expert_combine, grad_out [tokens, dim] of
    y's type; place and offsets of one lapsum_expert_order."""
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(y, "y")
    code = _dtype(y, "y")
    if y.dim() != 2:
        raise ValueError("y must be [rows, dim]")
    y = y.contiguous()
    dev = y.device
    _places(place, dev)
    _expect(weights, "weights", place.shape, torch.float32, dev)
    _expect(grad_out, "grad_out", (place.shape[0], y.shape[1]), y.dtype, dev)
    _offsets(offsets, offsets.numel() - 1, dev)
    grad_y = torch.empty_like(y)
    grad_w = torch.empty_like(weights)
    with _on_device(dev):
        _check(lib.lapsum_expert_combine_backward(
            _ptr(grad_out), _ptr(y), code, y.shape[0], y.shape[1], _ptr(weights), _ptr(place),
            _ptr(offsets), offsets.numel() - 1, place.shape[0], place.shape[1], _ptr(grad_y),
            _ptr(grad_w), _stream(dev)), "lapsum_expert_combine_backward")
    return grad_y, grad_w
