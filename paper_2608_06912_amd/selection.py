"""Binding of the hard selections of a language model: which experts a token
goes to, which continuations a beam search keeps, which entries of a key-value
cache stay.

As in the rest of the package the functions carry the C names
(include/lapsum.h has their definitions) and only check and marshal their
arguments.  The differentiable form of the routing is autograd.route_topk.

    w, idx = lapsum_route_forward(logits, 8, score="sigmoid", bias=bias,
                                  groups=8, topk_groups=4, group_top=2, renormalise=True)
    scores, tokens, parents = lapsum_beam_select(logits, beam_scores, num)
    lapsum_beam_reorder([k, v], parents, length=t)
    acc = lapsum_cache_accumulate(window_weights, kv_heads, seen=seen)
    k, v, acc, pos = lapsum_cache_evict(k, v, acc, seen, budget, sink=4, recent=64)
    slot = lapsum_cache_step(weights, k_new, v_new, seen, k, v, acc, pos, sink=4, recent=64)
"""
from __future__ import annotations

import ctypes

from . import _check, _on_device, _ptr, _stream, _torch, _workspace, load

__all__ = [
    "lapsum_route_forward_workspace_size", "lapsum_route_forward", "lapsum_route_backward",
    "lapsum_beam_select_workspace_size", "lapsum_beam_select", "lapsum_beam_reorder",
    "lapsum_cache_accumulate", "lapsum_cache_evict_workspace_size", "lapsum_cache_evict",
    "lapsum_cache_step",
]

_SCORES = {"softmax": 0, "sigmoid": 1}
_dtypes = None
_lib = None


class _BeamState(ctypes.Structure):
    """Mirror of lapsum_beam_state."""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("row_bytes", ctypes.c_int64),
                ("outer", ctypes.c_int64), ("outer_stride", ctypes.c_int64),
                ("live_bytes", ctypes.c_int64)]


def _load():
    """The library with the signatures of this module declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = load()
    vp, i64, f64, sz, i32 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t,
                             ctypes.c_int)
    lib.lapsum_route_forward_workspace_size.argtypes = [i64, i64, i64, i64, i32]
    lib.lapsum_route_forward_workspace_size.restype = sz
    lib.lapsum_route_forward.argtypes = [vp, i32, i64, i64, i64, i32, vp, i64, i64, i64, i64, i32,
                                         f64, vp, vp, vp, vp, sz, vp]
    lib.lapsum_route_forward.restype = i32
    lib.lapsum_route_backward.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, i64, i32, f64, vp, vp]
    lib.lapsum_route_backward.restype = i32
    lib.lapsum_beam_select_workspace_size.argtypes = [i64, i64, i64, i64]
    lib.lapsum_beam_select_workspace_size.restype = sz
    lib.lapsum_beam_select.argtypes = [vp, i32, i64, i64, i64, i64, vp, i64, vp, vp, vp, vp, sz, vp]
    lib.lapsum_beam_select.restype = i32
    lib.lapsum_beam_reorder.argtypes = [vp, i64, vp, i64, i64, i64, vp]
    lib.lapsum_beam_reorder.restype = i32
    lib.lapsum_cache_accumulate.argtypes = [vp, i32, i64, i64, i64, i64, i64, i64, i64, i64, vp, vp,
                                            vp, vp]
    lib.lapsum_cache_accumulate.restype = i32
    lib.lapsum_cache_evict_workspace_size.argtypes = [i64, i64, i64, i64]
    lib.lapsum_cache_evict_workspace_size.restype = sz
    lib.lapsum_cache_evict.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp, i64, i64, i64, i64, i64, i64,
                                       vp, vp, vp, vp, vp, sz, vp]
    lib.lapsum_cache_evict.restype = i32
    lib.lapsum_cache_step.argtypes = [vp, i32, i64, i64, vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, i64,
                                      i64, i64, i64, i64, i64, vp, vp]
    lib.lapsum_cache_step.restype = i32
    _lib = lib
    return lib


_native = None


def _node():
    """The calls in native code (csrc/selection_node.cpp), or False where only
    the library is built.  They take the common case and return None (or
    raise TypeError, for arguments of another type) for everything else, which
    then comes to the checks here."""
    global _native
    if _native is None:
        from .autograd import _load_node
        _native = _load_node()
    return _native


def _dtype(x, name):
    global _dtypes
    if _dtypes is None:
        torch = _torch()
        _dtypes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    code = _dtypes.get(x.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16")
    return code


def _device_tensor(x, name, dtype=None):
    torch = _torch()
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is not None and x.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}")
    return x


def _expect(x, name, shape, dtype, device, dense=True):
    """x, a tensor of this shape and type on `device`."""
    _device_tensor(x, name, dtype)
    if x.shape != shape or x.device != device:
        raise ValueError(f"{name} must have shape {tuple(shape)} on {device}")
    if dense and not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return x


def _may_write(x, name):
    """Refuse to write over what autograd would take for unchanged."""
    if x.requires_grad and _torch().is_grad_enabled():
        raise RuntimeError(f"{name} requires grad and is written in place, which has no gradient")


def _written(*tensors):
    """Tell autograd, which may have saved them, that these changed."""
    _torch().autograd.graph.increment_version(tensors)


def _count(value, name):
    if int(value) != value:
        raise ValueError(f"{name} must be an integer")
    return int(value)


def _row_view(x, name):
    """x as rows of its last dimension that are evenly apart: (tensor, rows,
    elements, stride)."""
    if x.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    n = x.shape[-1]
    if x.is_contiguous():
        return x, (x.numel() // n if n else 0), n, n
    if x.dim() != 2 or x.stride(1) != 1 or x.stride(0) < n:
        x = x.contiguous()
        return x, (x.numel() // n if n else 0), n, n
    return x, x.shape[0], n, x.stride(0)


# -------------------------------------------------------------- routing ----
def lapsum_route_forward_workspace_size(tokens: int, experts: int, top_k: int, groups: int = 1,
                                        with_counts: bool = False) -> int:
    return int(_load().lapsum_route_forward_workspace_size(tokens, experts, top_k, groups,
                                                           int(bool(with_counts))))


def lapsum_route_forward(logits, top_k: int, *, score: str = "softmax", bias=None, groups: int = 1,
                         topk_groups: int | None = None, group_top: int = 1,
                         renormalise: bool = False, scale: float = 1.0, counts: bool = False,
                         workspace=None):
    """The top_k experts of each token: logits [..., experts] (float32,
    bfloat16, float16), weights float32 and indices int32 [..., top_k], and
    with counts=True the tokens per expert, int32.  score "softmax" or
    "sigmoid"; bias: float32 [experts], added to the scores for the choice
    only.  A place without an expert has index -1 and weight 0."""
    node = _native or _node()
    if node and workspace is None and score in _SCORES:
        try:
            out = node.route(logits, top_k, _SCORES[score], bias, groups,
                             groups if topk_groups is None else topk_groups, group_top, renormalise,
                             scale, counts, False)
        except TypeError:
            out = None
        if out is not None:
            return tuple(out)
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(logits, "logits")
    code = _dtype(logits, "logits")
    x, tokens, experts, stride = _row_view(logits, "logits")
    if score not in _SCORES:
        raise ValueError(f"unknown score {score!r}")
    k = _count(top_k, "top_k")
    dev = x.device
    if bias is not None:
        _expect(bias, "bias", (experts,), torch.float32, dev)
    groups = _count(groups, "groups")
    topk_groups = groups if topk_groups is None else _count(topk_groups, "topk_groups")
    size = (*logits.shape[:-1], max(k, 0))
    weights = torch.empty(size, dtype=torch.float32, device=dev)
    indices = torch.empty(size, dtype=torch.int32, device=dev)
    count = ws = None
    nbytes = 0
    if counts:
        count = torch.empty(experts, dtype=torch.int32, device=dev)
        ws, nbytes = _workspace(lib.lapsum_route_forward_workspace_size(tokens, experts, k, groups, 1),
                                dev, workspace)
    with _on_device(dev):
        _check(lib.lapsum_route_forward(_ptr(x), code, tokens, experts, stride, _SCORES[score],
                                        _ptr(bias), groups, topk_groups, _count(group_top, "group_top"),
                                        k, int(bool(renormalise)), float(scale), _ptr(weights),
                                        _ptr(indices), _ptr(count), _ptr(ws), nbytes, _stream(dev)),
               "lapsum_route_forward")
    return (weights, indices, count) if counts else (weights, indices)


def lapsum_route_backward(grad_weights, logits, indices, *, score: str = "softmax",
                          renormalise: bool = False, scale: float = 1.0):
    """dL/dlogits of lapsum_route_forward's weights, in the logits' type and
    shape; logits, indices and options as they were in the forward."""
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(logits, "logits")
    code = _dtype(logits, "logits")
    x, tokens, experts, stride = _row_view(logits, "logits")
    if score not in _SCORES:
        raise ValueError(f"unknown score {score!r}")
    dev = x.device
    size = (*logits.shape[:-1], indices.shape[-1])
    _expect(indices, "indices", size, torch.int32, dev)
    _expect(grad_weights, "grad_weights", size, torch.float32, dev)
    grad = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    with _on_device(dev):
        _check(lib.lapsum_route_backward(_ptr(grad_weights), _ptr(x), code, tokens, experts, stride,
                                         _ptr(indices), _SCORES[score], size[-1],
                                         int(bool(renormalise)), float(scale), _ptr(grad),
                                         _stream(dev)), "lapsum_route_backward")
    return grad


# ---------------------------------------------------------- beam search ----
def lapsum_beam_select_workspace_size(batch: int, beams: int, vocab: int, num: int) -> int:
    return int(_load().lapsum_beam_select_workspace_size(batch, beams, vocab, num))


def lapsum_beam_select(logits, beam_scores, num: int, *, workspace=None):
    """The num best continuations of each request: logits [batch * beams,
    vocab] or [batch, beams, vocab], beam_scores float32 [batch, beams].
    Returns (scores, tokens, parents), each [batch, num]; score -inf, token -1
    and parent -1 where no continuation is left."""
    node = _native or _node()
    if node and workspace is None:
        try:
            out = node.beam_select(logits, beam_scores, num)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(logits, "logits")
    code = _dtype(logits, "logits")
    x, rows, vocab, stride = _row_view(logits, "logits")
    dev = x.device
    _device_tensor(beam_scores, "beam_scores", torch.float32)
    if beam_scores.dim() != 2 or not beam_scores.is_contiguous() or beam_scores.device != dev:
        raise ValueError(f"beam_scores must be contiguous [batch, beams] on {dev}")
    batch, beams = beam_scores.shape
    if rows != batch * beams:
        raise ValueError("logits must have batch * beams rows")
    num = _count(num, "num")
    scores = torch.empty((batch, max(num, 0)), dtype=torch.float32, device=dev)
    tokens = torch.empty((batch, max(num, 0)), dtype=torch.int32, device=dev)
    parents = torch.empty((batch, max(num, 0)), dtype=torch.int32, device=dev)
    ws, nbytes = _workspace(lib.lapsum_beam_select_workspace_size(batch, beams, vocab, num), dev,
                            workspace)
    with _on_device(dev):
        _check(lib.lapsum_beam_select(_ptr(x), code, batch, beams, vocab, stride, _ptr(beam_scores),
                                      num, _ptr(scores), _ptr(tokens), _ptr(parents), _ptr(ws),
                                      nbytes, _stream(dev)), "lapsum_beam_select")
    return scores, tokens, parents


def lapsum_beam_reorder(states, parents, *, length: int | None = None, out=None):
    """Move the rows of each state, [batch * beams, ...], to the beams they go
    on in: row (b, i) <- row (b, parents[b, i]).  length: of states
    [batch * beams, heads, room, dim] (any dimensions before room), move only
    the first `length` of room.  In place, or with `out` (as many tensors of
    the same shapes) into those; what is written must not be part of another
    state or out.  Returns the tensors written, which autograd
    takes as changed; in grad mode none of them may require grad."""
    states = list(states)
    outs = states if out is None else list(out)
    node = _native or _node()
    if node:
        try:
            if node.beam_reorder(states, parents, length, outs):
                return outs
        except TypeError:
            pass
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(parents, "parents", torch.int32)
    if parents.dim() != 2 or parents.stride(1) != 1 and parents.shape[1] > 1:
        raise ValueError("parents must be [batch, beams] with dense rows")
    batch, beams = parents.shape
    if len(outs) != len(states):
        raise ValueError("out must have one tensor for each state")
    dev = parents.device
    if not states or batch == 0:
        return outs
    if length is not None:
        length = _count(length, "length")
    array = (_BeamState * len(states))()
    for item, s, o in zip(array, states, outs):
        if not s.is_cuda or s.device != dev or s.dim() < 1 or s.shape[0] != batch * beams or \
                not s.is_contiguous():
            raise ValueError(f"a state must be contiguous with batch * beams rows on {dev}")
        if o is not s and (o.shape != s.shape or o.dtype is not s.dtype or o.device != dev
                           or not o.is_contiguous()):
            raise ValueError("out must be like the states")
        _may_write(o, "a state" if o is s else "out")
        size = s.element_size()
        row = s.stride(0) * size if s.shape[0] > 1 else s.numel() * size
        item.src, item.dst, item.row_bytes = s.data_ptr(), o.data_ptr(), row
        if length is None:
            item.outer, item.outer_stride, item.live_bytes = 1, row, row
        else:
            if s.dim() < 3 or not 0 <= length <= s.shape[-2]:
                raise ValueError("length needs states [rows, ..., room, dim] with room for it")
            piece = s.shape[-2] * s.shape[-1] * size
            item.outer = row // piece if piece else 0
            item.outer_stride, item.live_bytes = piece, length * s.shape[-1] * size
    with _on_device(dev):
        _check(lib.lapsum_beam_reorder(ctypes.addressof(array), len(states), _ptr(parents),
                                       parents.stride(0) if batch > 1 else beams, batch, beams,
                                       _stream(dev)), "lapsum_beam_reorder")
    _written(*outs)
    return outs


# ---------------------------------------------------------------- cache ----
def _strides3(x, name, written=False):
    """Byte strides of a cache [batch, kv_heads, slots, dim] with dense rows."""
    if x.dim() != 4 or (x.stride(3) != 1 and x.shape[3] > 1):
        raise ValueError(f"{name} must be [batch, kv_heads, slots, dim] with dense rows")
    size = x.element_size()
    sb, sh, ss, _ = x.stride()
    if written and any(s == 0 and n > 1 for s, n in zip(x.stride(), x.shape)):
        raise ValueError(f"{name} is written: its entries must not share memory")
    return (ctypes.c_int64 * 3)(sb * size, sh * size, ss * size)


def lapsum_cache_accumulate(weights, kv_heads: int, *, seen=None, acc=None):
    """Attention weight per cache entry: weights [batch, heads, queries, keys]
    summed over the query heads that share a key head and over the queries, to
    float32 [batch, kv_heads, keys].  seen (int32 [batch]): only the first
    seen[b] columns of a sequence count.  acc: added to, in place (in grad mode
    it may not require grad)."""
    node = _native or _node()
    if node:
        try:
            out = node.cache_accumulate(weights, kv_heads, seen, acc)
        except TypeError:
            out = None
        if out is not None:
            return out if acc is None else acc
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(weights, "weights")
    code = _dtype(weights, "weights")
    if weights.dim() != 4:
        raise ValueError("weights must be [batch, heads, queries, keys]")
    w = weights if weights.stride(3) == 1 or weights.shape[3] <= 1 else weights.contiguous()
    batch, heads, queries, keys = w.shape
    kv = _count(kv_heads, "kv_heads")
    dev = w.device
    if seen is not None:
        _expect(seen, "seen", (batch,), torch.int32, dev)
    if acc is None:
        out = torch.empty((batch, max(kv, 0), keys), dtype=torch.float32, device=dev)
    else:
        out = _expect(acc, "acc", (batch, kv, keys), torch.float32, dev)
        _may_write(acc, "acc")
    sb, sh, sq, _ = w.stride()
    with _on_device(dev):
        _check(lib.lapsum_cache_accumulate(_ptr(w), code, batch, heads, kv, queries, keys, sb, sh, sq,
                                           _ptr(seen), _ptr(acc), _ptr(out), _stream(dev)),
               "lapsum_cache_accumulate")
    if acc is not None:
        _written(acc)
    return out


def lapsum_cache_evict_workspace_size(batch: int, kv_heads: int, slots: int, budget: int) -> int:
    return int(_load().lapsum_cache_evict_workspace_size(batch, kv_heads, slots, budget))


def lapsum_cache_evict(k, v, acc, seen, budget: int, *, sink: int = 0, recent: int = 0, pos=None,
                       workspace=None):
    """The budget entries of each (sequence, head) that stay, as a new cache:
    k and v [batch, kv_heads, slots, dim] (one type, any outer strides), acc
    float32 [batch, kv_heads, slots], seen int32 [batch], and pos int32 like
    acc where slots do not hold their own positions.  Returns (k, v, acc, pos)
    with `budget` slots; where fewer stay, zeros and position -1 follow."""
    node = _native or _node()
    if node and workspace is None:
        try:
            out = node.cache_evict(k, v, acc, seen, budget, sink, recent, pos)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(k, "k")
    _device_tensor(v, "v")
    ks, vs = _strides3(k, "k"), _strides3(v, "v")
    batch, kv, slots, dim = k.shape
    dev = k.device
    if v.shape != k.shape or v.dtype is not k.dtype or v.device != dev:
        raise ValueError("k and v must be alike")
    _expect(acc, "acc", (batch, kv, slots), torch.float32, dev)
    _expect(seen, "seen", (batch,), torch.int32, dev)
    if pos is not None:
        _expect(pos, "pos", (batch, kv, slots), torch.int32, dev)
    budget = _count(budget, "budget")
    size = (batch, kv, max(budget, 0), dim)
    k_out = torch.empty(size, dtype=k.dtype, device=dev)
    v_out = torch.empty(size, dtype=k.dtype, device=dev)
    acc_out = torch.empty(size[:3], dtype=torch.float32, device=dev)
    pos_out = torch.empty(size[:3], dtype=torch.int32, device=dev)
    ws, nbytes = _workspace(lib.lapsum_cache_evict_workspace_size(batch, kv, slots, budget), dev,
                            workspace)
    with _on_device(dev):
        _check(lib.lapsum_cache_evict(_ptr(k), ks, _ptr(v), vs, dim * k.element_size(), _ptr(acc),
                                      _ptr(pos), _ptr(seen), batch, kv, slots, budget,
                                      _count(sink, "sink"), _count(recent, "recent"), _ptr(k_out),
                                      _ptr(v_out), _ptr(acc_out), _ptr(pos_out), _ptr(ws), nbytes,
                                      _stream(dev)), "lapsum_cache_evict")
    return k_out, v_out, acc_out, pos_out


def lapsum_cache_step(weights, k_new, v_new, seen, k, v, acc, pos, *, sink: int = 0, recent: int = 1):
    """One generated token, in place: acc += weights [batch, heads, slots] (or
    [batch, heads, 1, slots]) summed over the heads that share a key head;
    then k_new, v_new [batch, kv_heads, dim] (or [batch, kv_heads, 1, dim])
    take the first empty slot (pos -1) or that of the smallest acc outside the
    first `sink` and last `recent` positions, at position seen[b].  Returns the slots, int32
    [batch, kv_heads].  The caller advances seen.  Autograd takes k, v, acc and
    pos as changed; in grad mode none of them may require grad."""
    node = _native or _node()
    if node:
        try:
            out = node.cache_step(weights, k_new, v_new, seen, k, v, acc, pos, sink, recent)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    _device_tensor(weights, "weights")
    code = _dtype(weights, "weights")
    _device_tensor(k, "k")
    _device_tensor(v, "v")
    ks, vs = _strides3(k, "k", True), _strides3(v, "v", True)
    batch, kv, slots, dim = k.shape
    dev = k.device
    if v.shape != k.shape or v.dtype is not k.dtype or v.device != dev or weights.device != dev:
        raise ValueError("k and v must be alike, and the weights on their device")
    w = weights
    if w.dim() == 4 and w.shape[2] == 1:
        w = w[:, :, 0]
    if w.dim() != 3 or w.shape[0] != batch or w.shape[2] != slots:
        raise ValueError("weights must be [batch, heads, slots]")
    if w.stride(2) != 1 and slots > 1:
        w = w.contiguous()
    rows = []
    for name, x in (("k_new", k_new), ("v_new", v_new)):
        _device_tensor(x, name, k.dtype)
        if x.dim() == 4 and x.shape[2] == 1:
            x = x[:, :, 0]
        if x.shape != (batch, kv, dim) or x.device != dev:
            raise ValueError(f"{name} must be [batch, kv_heads, dim] on {dev}")
        rows.append(x if x.is_contiguous() else x.contiguous())
    _expect(acc, "acc", (batch, kv, slots), torch.float32, dev)
    _expect(pos, "pos", (batch, kv, slots), torch.int32, dev)
    _expect(seen, "seen", (batch,), torch.int32, dev)
    for name, x in (("k", k), ("v", v), ("acc", acc)):
        _may_write(x, name)
    slot = torch.empty((batch, kv), dtype=torch.int32, device=dev)
    with _on_device(dev):
        _check(lib.lapsum_cache_step(_ptr(w), code, w.stride(0), w.stride(1), _ptr(rows[0]),
                                     _ptr(rows[1]), _ptr(seen), _ptr(k), ks, _ptr(v), vs,
                                     dim * k.element_size(), _ptr(acc), _ptr(pos), batch, w.shape[1],
                                     kv, slots, _count(sink, "sink"), _count(recent, "recent"),
                                     _ptr(slot), _stream(dev)), "lapsum_cache_step")
    _written(k, v, acc, pos)
    return slot
