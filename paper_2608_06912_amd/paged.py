"""Binding of the key-value cache in pages: new entries written, as they are or in
8 bits, read back, and attended to by one new token per sequence.

The functions carry the C names (include/lapsum.h has their definitions) and only
check and marshal their arguments.

    k = torch.empty(pages, kv_heads, slots, dim, dtype=torch.int8, device="cuda")   # v alike
    k_scale = torch.empty(pages, kv_heads, slots, device="cuda")
    lapsum_cache_append(k_new, v_new, seen, k, v, table=table, k_scale=k_scale, v_scale=v_scale)
    y = lapsum_cache_attend(q, k, v, seen + 1, table=table, k_scale=k_scale, v_scale=v_scale)

Without a table the cache is [batch, kv_heads, slots, dim], as
lapsum_cache_evict returns it; the attention's weights are then what
lapsum_cache_step takes.

None of this is differentiable.  Entries are written without their history, and what
is read back or attended to from inputs that require grad, in grad mode, raises where its
gradient is asked for.
"""
from __future__ import annotations

import ctypes
import math

from . import _check, _on_device, _ptr, _stream, _torch, _workspace, load
from .selection import _count, _device_tensor, _dtype, _expect, _may_write, _node, _written

__all__ = [
    "lapsum_cache_append", "lapsum_cache_read", "lapsum_cache_attend_workspace_size",
    "lapsum_cache_attend",
]

_lib = None


class _Paged(ctypes.Structure):
    """Mirror of lapsum_paged."""
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("pages", ctypes.c_int64),
                ("slots", ctypes.c_int64), ("stride_page", ctypes.c_int64),
                ("stride_head", ctypes.c_int64), ("stride_slot", ctypes.c_int64),
                ("scale_stride_page", ctypes.c_int64), ("scale_stride_head", ctypes.c_int64)]


def _load():
    """The library with the signatures of this module declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = load()
    vp, i64, f64, sz, i32 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t,
                             ctypes.c_int)
    cache = ctypes.POINTER(_Paged)
    lib.lapsum_cache_append.argtypes = [vp, vp, vp, vp, i32, i64, i64, i64, i64, vp, vp, cache, cache,
                                        i32, vp, i64, vp]
    lib.lapsum_cache_append.restype = i32
    lib.lapsum_cache_read.argtypes = [cache, i32, i64, i64, i64, i64, vp, vp, i64, vp, i32, vp]
    lib.lapsum_cache_read.restype = i32
    lib.lapsum_cache_attend_workspace_size.argtypes = [i64, i64, i64, i64, i64, i64]
    lib.lapsum_cache_attend_workspace_size.restype = sz
    lib.lapsum_cache_attend.argtypes = [vp, i64, i64, i32, cache, cache, i32, i64, i64, i64, i64, vp, vp,
                                        i64, f64, i64, vp, vp, vp, vp, sz, vp]
    lib.lapsum_cache_attend.restype = i32
    _lib = lib
    return lib


def _kind(x, name):
    torch = _torch()
    if x.dtype is torch.int8:
        return 3
    if x.dtype is torch.float8_e4m3fn:
        return 4
    try:
        return _dtype(x, name)
    except ValueError:
        raise ValueError(f"{name} must be float32, bfloat16, float16, int8 or float8_e4m3fn") from None


def _cache(x, scale, name, written=False):
    """lapsum_paged of a cache [pages, kv_heads, slots, dim] with dense rows."""
    torch = _torch()
    _device_tensor(x, name)
    kind = _kind(x, name)
    if x.dim() != 4 or (x.stride(3) != 1 and x.shape[3] > 1):
        raise ValueError(f"{name} must be [pages, kv_heads, slots, dim] with dense rows")
    if written and any(s == 0 and n > 1 for s, n in zip(x.stride(), x.shape)):
        raise ValueError(f"{name} is written: its entries must not share memory")
    c = _Paged(x.data_ptr(), None, x.shape[0], x.shape[2], *x.stride()[:3], 0, 0)
    if (kind >= 3) != (scale is not None):
        raise ValueError(f"{name} needs a scale if it is in 8 bits, and only then")
    if scale is not None:
        _expect(scale, f"{name}_scale", x.shape[:3], torch.float32, x.device, dense=False)
        if scale.stride(2) != 1 and x.shape[2] > 1:
            raise ValueError(f"{name}_scale must have dense slots")
        if written and any(s == 0 and n > 1 for s, n in zip(scale.stride(), scale.shape)):
            raise ValueError(f"{name}_scale is written: its entries must not share memory")
        c.scale, c.scale_stride_page, c.scale_stride_head = scale.data_ptr(), scale.stride(0), scale.stride(1)
    return c, kind


def _table(table, batch, device):
    """(address of the contiguous table or None, width)."""
    if table is None:
        return None, 0
    _device_tensor(table, "table", _torch().int32)
    if table.dim() != 2 or table.shape[0] != batch or not table.is_contiguous() or table.device != device:
        raise ValueError(f"table must be contiguous [batch, pages] on {device}")
    # (one without pages has no address, and is not to be taken for none)
    return table.data_ptr() or _ALIGNED, table.shape[1]


_ALIGNED = 256   # an address that is never read


def _pair(k, v, k_scale, v_scale, written=False):
    ck, kind = _cache(k, k_scale, "k", written)
    cv, _ = _cache(v, v_scale, "v", written)
    if v.shape != k.shape or v.dtype is not k.dtype or v.device != k.device:
        raise ValueError("k and v must be alike")
    return ck, cv, kind


def _no_gradient(outs, inputs, where):
    """outs, such that asking for a gradient through them is an error, if autograd would
    record a call with these inputs."""
    torch = _torch()
    if not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in inputs):
        return outs
    error = torch._C._functions.DelayedError(f"{where} has no gradient".encode(), len(outs))
    found = error(*[t.detach().requires_grad_() for t in outs])
    return [found] if isinstance(found, torch.Tensor) else list(found)


def lapsum_cache_append(k_new, v_new, seen, k, v, *, table=None, count=None, k_scale=None, v_scale=None):
    """Write new entries into a cache, in place: entry i of sequence b, k_new and v_new
    [batch, kv_heads, new, dim] (or [batch, kv_heads, dim], one each), at position
    seen[b] + i, for i < count[b] (int32 [batch]; None: all).  k and v
    [pages, kv_heads, slots, dim] of the entries' type, int8 or float8_e4m3fn,
    those with float32 scales [pages, kv_heads, slots]; table int32 [batch, pages of
    a sequence], None where page b is sequence b's.  Positions without a page are
    not written.  The caller advances seen.  k may be v, for a cache that is both, where
    k_new is v_new.  Autograd takes k, v and the scales as changed; in grad mode none of
    them may require grad.  No gradient goes back to k_new and v_new."""
    node = _node()
    if node:
        try:
            if node.cache_append(k_new, v_new, seen, k, v, table, count, k_scale, v_scale):
                return
        except TypeError:
            pass
    torch = _torch()
    lib = _lib or _load()
    ck, cv, kind = _pair(k, v, k_scale, v_scale, True)
    dev = k.device
    rows = []
    for name, x in (("k_new", k_new), ("v_new", v_new)):
        _device_tensor(x, name)
        x = x[:, :, None] if x.dim() == 3 else x
        if x.dim() != 4 or x.shape[1] != k.shape[1] or x.shape[3] != k.shape[3] or x.device != dev:
            raise ValueError(f"{name} must be [batch, kv_heads, new, dim] on {dev}")
        if x.stride(3) != 1 and x.shape[3] > 1:
            x = x.contiguous()
        rows.append(x)
    kn, vn = rows
    if vn.shape != kn.shape or vn.dtype is not kn.dtype:
        raise ValueError("k_new and v_new must be alike")
    code = _dtype(kn, "k_new")
    if kind < 3 and kind != code:
        raise ValueError("a cache that is not in 8 bits must have its entries' type")
    batch, kv, fresh, dim = kn.shape
    _expect(seen, "seen", (batch,), torch.int32, dev)
    if count is not None:
        _expect(count, "count", (batch,), torch.int32, dev)
    table, width = _table(table, batch, dev)
    out = [t for t in (k, v, k_scale, v_scale) if t is not None]
    for x in out:
        _may_write(x, "a cache")
    with _on_device(dev):
        _check(lib.lapsum_cache_append(_ptr(kn), (ctypes.c_int64 * 3)(*kn.stride()[:3]), _ptr(vn),
                                       (ctypes.c_int64 * 3)(*vn.stride()[:3]), code, batch, kv, fresh,
                                       dim, _ptr(seen), _ptr(count), ctypes.byref(ck),
                                       ctypes.byref(cv), kind, table, width, _stream(dev)),
               "lapsum_cache_append")
    _written(*out)


def lapsum_cache_read(x, lens, room: int, *, table=None, scale=None, dtype=None):
    """A cache's entries by sequence: [batch, kv_heads, room, dim], positions from
    lens[b] (int32 [batch]) on and those without a page 0.  x, table and scale as in
    lapsum_cache_append; dtype: the cache's own, or for one in 8 bits float32,
    bfloat16 or float16 (float32 if None).  Not differentiable: a gradient through it
    is an error."""
    node = _node()
    if node:
        try:
            out = node.cache_read(x, lens, room, table, scale, dtype)
        except TypeError:
            out = None
        if out is not None:
            return out
    torch = _torch()
    lib = _lib or _load()
    c, kind = _cache(x, scale, "x")
    dev = x.device
    _device_tensor(lens, "lens", torch.int32)
    batch = lens.numel()
    _expect(lens, "lens", (batch,), torch.int32, dev)
    table, width = _table(table, batch, dev)
    room = _count(room, "room")
    if dtype is None:
        dtype = torch.float32 if kind >= 3 else x.dtype
    if kind < 3 and dtype is not x.dtype:
        raise ValueError("a cache that is not in 8 bits is read back in its own type")
    out = torch.empty((batch, x.shape[1], max(room, 0), x.shape[3]), dtype=dtype, device=dev)
    with _on_device(dev):
        _check(lib.lapsum_cache_read(ctypes.byref(c), kind, batch, x.shape[1], room, x.shape[3],
                                     _ptr(lens), table, width, _ptr(out), _dtype(out, "dtype"),
                                     _stream(dev)), "lapsum_cache_read")
    return _no_gradient([out], (x, scale), "lapsum_cache_read")[0]


def lapsum_cache_attend_workspace_size(batch: int, heads: int, kv_heads: int, dim: int, room: int,
                                       window: int = 0) -> int:
    return int(_load().lapsum_cache_attend_workspace_size(batch, heads, kv_heads, dim, room, window))


def lapsum_cache_attend(q, k, v, lens, *, table=None, k_scale=None, v_scale=None, scale=None,
                        window: int = 0, lse: bool = False, weights: bool = False, workspace=None):
    """Attention of one new token per sequence, q [batch, heads, dim] (or [batch,
    heads, 1, dim]), over the first lens[b] (int32 [batch]) entries of its cache:
    out like q.  k, v, table and scales as in lapsum_cache_append; heads a
    multiple of kv_heads; scale of the scores: dim ** -0.5 if None; window > 0:
    only the last `window` entries.  lse=True adds the log-sum-exp of the
    scores, float32 [batch, heads]; weights=True the weights, float32
    [batch, heads, room] (room: the slots of the table's pages).  A sequence
    without entries gets zeros, and lse -inf.  Not differentiable: a gradient through
    it is an error."""
    node = _node()
    if node and workspace is None:
        try:
            out = node.cache_attend(q, k, v, lens, table, k_scale, v_scale, scale, window, lse, weights)
        except TypeError:
            out = None
        if out is not None:
            return out[0] if len(out) == 1 else tuple(out)
    torch = _torch()
    lib = _lib or _load()
    ck, cv, kind = _pair(k, v, k_scale, v_scale)
    dev = k.device
    _device_tensor(q, "q")
    code = _dtype(q, "q")
    shape = q.shape
    if q.dim() == 4 and q.shape[2] == 1:
        q = q[:, :, 0]
    if q.dim() != 3 or q.device != dev or q.shape[2] != k.shape[3]:
        raise ValueError(f"q must be [batch, heads, dim] on {dev}")
    if q.stride(2) != 1 and q.shape[2] > 1:
        q = q.contiguous()
    if kind < 3 and kind != code:
        raise ValueError("a cache that is not in 8 bits must have the queries' type")
    batch, heads, dim = q.shape
    kv = k.shape[1]
    if not kv or heads % kv:
        raise ValueError("heads must be a multiple of kv_heads")
    _expect(lens, "lens", (batch,), torch.int32, dev)
    table, width = _table(table, batch, dev)
    room = k.shape[2] if table is None else width * k.shape[2]
    window = _count(window, "window")
    scale = dim ** -0.5 if scale is None else float(scale)
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    out = torch.empty(shape, dtype=q.dtype, device=dev)
    total = torch.empty((batch, heads), dtype=torch.float32, device=dev) if lse or weights else None
    w = torch.empty((batch, heads, room), dtype=torch.float32, device=dev) if weights else None
    ws, nbytes = _workspace(lib.lapsum_cache_attend_workspace_size(batch, heads, kv, dim, room, window),
                            dev, workspace)
    with _on_device(dev):
        _check(lib.lapsum_cache_attend(_ptr(q), q.stride(0), q.stride(1), code, ctypes.byref(ck),
                                       ctypes.byref(cv), kind, batch, heads, kv, dim, _ptr(lens),
                                       table, width, scale, window, _ptr(out), _ptr(total),
                                       _ptr(w), _ptr(ws), nbytes, _stream(dev)), "lapsum_cache_attend")
    found = [out] + ([total] if lse else []) + ([w] if weights else [])
    found = _no_gradient(found, (q, k, v, k_scale, v_scale), "lapsum_cache_attend")
    return found[0] if len(found) == 1 else tuple(found)
