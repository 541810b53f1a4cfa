"""The products and reads that follow a language model's hard selections, as
measured cases: the products of the experts that a router chose, and the
key-value cache that holds what a sequence has seen.

A case names its path (`op`):

  "append"   cache_append: new keys and values into the pages of their sequences,
             as they are or quantised to 8 bits by row
  "read"     cache_read: a paged cache read back as one array per sequence
  "attend"   cache_attend: one new token's attention over the cache of each
             sequence, paged or not, with the weights and log-sum-exp if asked
  "product"  expert_matmul: rows times the matrices of their experts; with
             `train` also the gradients of rows and matrices
  "combine"  expert_order and expert_combine: the order of the chosen experts,
             and their outputs summed by the router's weights; with `train` also
             the gradients of outputs and weights

A cache is [pages, kv_heads, page, dim] with a table of pages per sequence, or
[batch, kv_heads, slots, dim] without one.  A row in 8 bits has a scale: its
largest magnitude over 127 (int8) or 448 (e4m3).
"""
import math

import torch

own = False

DEV = "cuda"
MOST = {"int8": 127.0, "float8_e4m3fn": 448.0}
TINY = 2.0 ** -126


# ---------------------------------------------------------------- cases ----
def listed():
    return [
        # the keys and values of one decode step of 64 requests: latency
        {"name": "append_step", "op": "append", "batch": 64, "kv": 8, "dim": 128, "new": 1,
         "ragged": False, "seen": 2000, "page": 16, "paged": True, "dtype": "bfloat16",
         "cache": "int8"},
        # a batch of prompts of different lengths
        {"name": "append_prompts", "op": "append", "batch": 12, "kv": 8, "dim": 128, "new": 8192,
         "ragged": True, "seen": 0, "page": 64, "paged": True, "dtype": "bfloat16",
         "cache": "float8_e4m3fn"},
        # one short sequence back in 16 bits, an odd page and dimension
        {"name": "read_short", "op": "read", "batch": 1, "kv": 4, "dim": 80, "len_min": 1003,
         "len_max": 1003, "page": 24, "paged": True, "cache": "int8", "dtype": "float16"},
        # a long batch back, as for the attention of many new tokens at once
        {"name": "read_long", "op": "read", "batch": 8, "kv": 8, "dim": 128, "len_min": 8000,
         "len_max": 32768, "page": 64, "paged": True, "cache": "float8_e4m3fn", "dtype": "bfloat16"},
        # one request's next token
        {"name": "attend_one", "op": "attend", "batch": 1, "heads": 32, "kv": 8, "dim": 128,
         "len_min": 4099, "len_max": 4099, "page": 16, "paged": True, "window": 0,
         "dtype": "bfloat16", "cache": "bfloat16", "lse": False, "weights": False},
        # 64 requests' next token: ragged lengths, 8 bits
        {"name": "attend_batch", "op": "attend", "batch": 64, "heads": 32, "kv": 8, "dim": 128,
         "len_min": 1, "len_max": 8192, "page": 32, "paged": True, "window": 0,
         "dtype": "bfloat16", "cache": "int8", "lse": False, "weights": False},
        # four long contexts
        {"name": "attend_long", "op": "attend", "batch": 4, "heads": 64, "kv": 8, "dim": 128,
         "len_min": 100003, "len_max": 131072, "page": 64, "paged": True, "window": 0,
         "dtype": "bfloat16", "cache": "bfloat16", "lse": True, "weights": False},
        # one decode step of 16 requests: few rows, each with matrices of its own
        {"name": "product_step", "op": "product", "tokens": 16, "top_k": 4, "experts": 64,
         "in": 2048, "out": 1024, "layout": "in_out", "gather": True, "dropped": 0.0,
         "dtype": "bfloat16", "train": False},
        # a packed prompt through many experts
        {"name": "product_prompt", "op": "product", "tokens": 16384, "top_k": 8, "experts": 128,
         "in": 2048, "out": 1536, "layout": "out_in", "gather": True, "dropped": 0.0,
         "dtype": "float16", "train": False},
        # a training step's layer, some places without an expert
        {"name": "product_train", "op": "product", "tokens": 8192, "top_k": 2, "experts": 8,
         "in": 2048, "out": 4096, "layout": "in_out", "gather": True, "dropped": 0.02,
         "dtype": "bfloat16", "train": True},
        # the order and the sum of that decode step: latency
        {"name": "combine_step", "op": "combine", "tokens": 16, "top_k": 4, "experts": 64,
         "dim": 2048, "dropped": 0.0, "dtype": "bfloat16", "train": False},
        # the same for a training step
        {"name": "combine_train", "op": "combine", "tokens": 16384, "top_k": 8, "experts": 128,
         "dim": 2048, "dropped": 0.02, "dtype": "bfloat16", "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / 4e14)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _drawn(rng)
        if _cost(case) <= most:
            return case


def _drawn(rng):
    op = rng.choice(["append", "read", "attend", "attend", "product", "product", "combine"])
    floats = ["float32", "bfloat16", "float16"]
    dtype = rng.choice(floats)
    if op in ("product", "combine"):
        experts = _log_int(rng, 2, 256)
        top_k = rng.randint(1, min(8, experts))
        tokens = _log_int(rng, 1, 32768)
        case = {"op": op, "tokens": tokens, "top_k": top_k, "experts": experts}
        more = {"dropped": rng.choice([0.0, 0.0, 0.05]), "dtype": dtype, "train": rng.random() < 0.5}
        if op == "combine":
            return {**case, "dim": 8 * _log_int(rng, 8, 512) + rng.choice([0, 0, 0, 1]), **more}
        # widths that are whole vectors mostly, and some that are not
        n_in, n_out = (8 * _log_int(rng, 8, 512) + rng.choice([0, 0, 0, 0, 3]) for _ in range(2))
        if experts * n_in * n_out > 1 << 29:
            experts = case["experts"] = max(2, (1 << 29) // (n_in * n_out))
            case["top_k"] = min(top_k, experts)
        return {**case, "in": n_in, "out": n_out, "layout": rng.choice(["in_out", "out_in"]),
                "gather": rng.random() < 0.7, **more}
    kv, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 256])
    cache = rng.choice([dtype, "int8", "float8_e4m3fn"])
    paged = rng.random() < 0.75
    case = {"op": op, "kv": kv, "dim": dim, "paged": paged,
            "page": rng.choice([8, 16, 24, 32, 64, 128, 256]), "dtype": dtype, "cache": cache}
    if op == "append":
        new = _log_int(rng, 1, 16384)
        batch = _log_int(rng, 1, max(1, min(256, (1 << 27) // (new * kv * dim))))
        return {**case, "batch": batch, "new": new, "ragged": rng.random() < 0.5,
                "seen": rng.choice([0, rng.randint(1, 3000)])}
    len_max = _log_int(rng, 1, 131072)
    batch = _log_int(rng, 1, max(1, min(128, (1 << 28) // (len_max * kv * dim))))
    case.update(batch=batch, len_max=len_max, len_min=max(1, int(len_max * rng.uniform(0.05, 1.0))))
    if op == "read":
        return case
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8, 16])
    return {**case, "heads": heads, "window": rng.choice([0, 0, 0, rng.randint(1, len_max)]),
            "lse": rng.random() < 0.5,
            "weights": batch * heads * len_max <= 1 << 25 and rng.random() < 0.4}


# --------------------------------------------------------------- inputs ----
def _lengths(c):
    """A batch's sequence lengths: from the shortest to the longest, evenly."""
    lo, hi, batch = c["len_min"], c["len_max"], c["batch"]
    return [hi] if batch == 1 else [lo + (hi - lo) * i // (batch - 1) for i in range(batch)]


def _counts(c):
    """The new entries of each sequence of an append."""
    n, batch = c["new"], c["batch"]
    return [n - (n - 1) * i // batch if c["ragged"] else n for i in range(batch)]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages(c, lengths, gen):
    """(leading size of the cache, slots of a page, table or None): pages in any
    order, a few of them free; entries of the table past a sequence's end are -1."""
    if not c["paged"]:
        return c["batch"], max(lengths), None
    page = c["page"]
    need = torch.tensor([-(-n // page) for n in lengths], device=DEV)
    total, width = sum(-(-n // page) for n in lengths), -(-max(lengths) // page)
    free = torch.randperm(total + 3, generator=gen, device=DEV)
    first = need.cumsum(0) - need
    at = torch.arange(width, device=DEV)
    table = free[(first[:, None] + at).clamp(max=total - 1)]
    return total + 3, page, torch.where(at < need[:, None], table, -1).to(torch.int32)


def _cache(c, size, gen):
    """A filled cache and its scales (None where it is not quantised)."""
    if c["cache"] not in MOST:
        return torch.randn(size, generator=gen, device=DEV, dtype=getattr(torch, c["cache"])), None
    x = torch.randn(size, generator=gen, device=DEV, dtype=torch.float16).mul_(0.28 * MOST[c["cache"]])
    x = x.clamp_(-MOST[c["cache"]], MOST[c["cache"]])
    x = x.round_().to(torch.int8) if c["cache"] == "int8" else x.to(torch.float8_e4m3fn)
    scale = torch.rand(size[:3], generator=gen, device=DEV).add_(0.5).mul_(3.5 / MOST[c["cache"]])
    return x, scale


def _prepare_append(c, gen):
    counts = _counts(c)
    ends = [c["seen"] + n for n in counts]
    pages, page, table = _pages(c, ends, gen)
    s = {"table": table, "seen": _int32([c["seen"]] * c["batch"]),
         "count": _int32(counts) if c["ragged"] else None}
    kind = getattr(torch, c["dtype"])
    for n in ("k", "v"):
        x = torch.randn(c["batch"], c["kv"], c["new"], c["dim"], generator=gen, device=DEV)
        # some channels are larger than the others
        x *= 0.5 + 2.0 * torch.rand(c["kv"], 1, c["dim"], generator=gen, device=DEV).pow_(4.0)
        s[n + "_new"] = x.to(kind)
        s[n], s[n + "_scale"] = _cache(c, (pages, c["kv"], page, c["dim"]), gen)
    return s


def _prepare_read(c, gen):
    lengths = _lengths(c)
    pages, page, table = _pages(c, lengths, gen)
    x, scale = _cache(c, (pages, c["kv"], page, c["dim"]), gen)
    return {"x": x, "scale": scale, "table": table, "lens": _int32(lengths)}


def _prepare_attend(c, gen):
    lengths = _lengths(c)
    pages, page, table = _pages(c, lengths, gen)
    s = {"table": table, "lens": _int32(lengths)}
    q = 1.5 * torch.randn(c["batch"], c["heads"], c["dim"], generator=gen, device=DEV)
    s["q"] = q.to(getattr(torch, c["dtype"]))
    for n in ("k", "v"):
        s[n], s[n + "_scale"] = _cache(c, (pages, c["kv"], page, c["dim"]), gen)
    return s


def _chosen(c, gen):
    """The router's choice, int32 [tokens, top_k]: some experts are liked more
    than others, and a share of the places has no expert (-1)."""
    x = torch.randn(c["tokens"], c["experts"], generator=gen, device=DEV)
    x += 0.5 * torch.randn(c["experts"], generator=gen, device=DEV)
    at = torch.topk(x, c["top_k"]).indices.to(torch.int32)
    none = torch.rand(at.shape, generator=gen, device=DEV) < c["dropped"]
    return at.masked_fill_(none, -1)


def _prepare_product(c, gen):
    order, place, offsets = _order(_chosen(c, gen), c["experts"])
    kind = getattr(torch, c["dtype"])
    rows = c["tokens"] * c["top_k"]
    size = (c["tokens"] if c["gather"] else rows, c["in"])
    e, a, b = c["experts"], c["in"], c["out"]
    w = torch.randn((e, b, a) if c["layout"] == "out_in" else (e, a, b), generator=gen, device=DEV,
                    dtype=kind).mul_(a ** -0.5)
    x = torch.randn(size, generator=gen, device=DEV).to(kind).requires_grad_(c["train"])
    s = {"w": w.requires_grad_(c["train"]), "x": x, "offsets": offsets,
         "ends": offsets.tolist(), "order": order, "place": place}
    if c["train"]:
        s["g"] = torch.randn(rows, b, generator=gen, device=DEV).to(kind)
    return s


def _prepare_combine(c, gen):
    kind = getattr(torch, c["dtype"])
    y = torch.randn(c["tokens"] * c["top_k"], c["dim"], generator=gen, device=DEV).to(kind)
    w = torch.rand(c["tokens"], c["top_k"], generator=gen, device=DEV).add_(0.1)
    w /= w.sum(-1, keepdim=True)
    s = {"at": _chosen(c, gen), "y": y.requires_grad_(c["train"]), "w": w.requires_grad_(c["train"])}
    if c["train"]:
        s["g"] = torch.randn(c["tokens"], c["dim"], generator=gen, device=DEV).to(kind)
    return s


_PREPARE = {"append": _prepare_append, "read": _prepare_read, "attend": _prepare_attend,
            "product": _prepare_product, "combine": _prepare_combine}


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 57)
    return {"case": case, **_PREPARE[case["op"]](case, gen)}


# ---------------------------------------------------------- plain forms ----
def _quantised(x, kind):
    """Codes and scales of rows, in 32 bits."""
    x = x.float()
    scale = (x.abs().amax(-1) / MOST[kind]).clamp(min=TINY)
    y = x / scale[..., None]
    return (y.round().to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)), scale


def _plain_append(s):
    c = s["case"]
    at = s["seen"].long()[:, None] + torch.arange(c["new"], device=DEV)   # positions
    if s["table"] is None:
        page, slot = torch.arange(c["batch"], device=DEV)[:, None].expand_as(at), at
    else:
        width = s["table"].shape[1]
        page = s["table"].long().gather(1, (at // c["page"]).clamp(max=width - 1))
        slot = at % c["page"]
    if s["count"] is not None:
        here = torch.arange(c["new"], device=DEV) < s["count"][:, None]
        page, slot = page[here], slot[here]
    for n in ("k", "v"):
        x = s[n + "_new"].transpose(1, 2)                                 # [batch, new, kv, dim]
        x = x if s["count"] is None else x[here]
        if c["cache"] in MOST:
            x, scale = _quantised(x, c["cache"])
            s[n + "_scale"][page, :, slot] = scale
            s[n].view(torch.int8)[page, :, slot] = x.view(torch.int8)
        else:
            s[n][page, :, slot] = x
    return [s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None]


def _whole(x, scale, table, room):
    """A cache as float32 [batch, kv, room, dim], entries past the end whatever they are."""
    if table is not None:
        at = table.long().clamp(min=0)
        if x.dtype == torch.float8_e4m3fn:
            x = x.view(torch.int8)[at].view(torch.float8_e4m3fn)
        else:
            x = x[at]
        x = x.transpose(1, 2).flatten(2, 3)[:, :, :room]
        scale = None if scale is None else scale[at].transpose(1, 2).flatten(2, 3)[:, :, :room]
    x = x.float()
    return x if scale is None else x * scale[..., None]


def _plain_read(s):
    c = s["case"]
    x = _whole(s["x"], s["scale"], s["table"], c["len_max"])
    gone = torch.arange(c["len_max"], device=DEV) >= s["lens"][:, None]
    return x.masked_fill(gone[:, None, :, None], 0.0).to(getattr(torch, c["dtype"]))


def _plain_attend(s):
    c = s["case"]
    room = c["len_max"] if s["table"] is None else s["table"].shape[1] * c["page"]
    k = _whole(s["k"], s["k_scale"], s["table"], room)
    at = torch.arange(room, device=DEV)
    lens = s["lens"].long()[:, None]
    gone = (at >= lens) | (at < lens - (c["window"] or room))
    q = s["q"].float().view(c["batch"], c["kv"], -1, c["dim"]) * c["dim"] ** -0.5
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).masked_fill_(gone[:, None, None], -math.inf)
    del k
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    w = e / total
    v = _whole(s["v"], s["v_scale"], s["table"], room)
    y = torch.matmul(w, v.masked_fill(gone[:, None, :, None], 0.0)).flatten(1, 2).to(s["q"].dtype)
    out = [y]
    if c["lse"]:
        out.append((top + torch.log(total)).flatten(1))
    if c["weights"]:
        out.append(w.flatten(1, 2))
    return out


def _order(at, experts):
    """The places [tokens * top_k] by expert, those without one last; each
    place's position in that order (-1 without an expert); each expert's first
    position and the end."""
    key = torch.where((at >= 0) & (at < experts), at, experts).reshape(-1).long()
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=DEV))
    place = place.masked_fill_(key == experts, -1)
    count = torch.zeros(experts + 1, dtype=torch.int64, device=DEV)
    count.scatter_add_(0, key, torch.ones_like(key))
    ends = count[:experts].cumsum(0)
    offsets = torch.cat([ends[:1] * 0, ends])
    return order.int(), place.view(at.shape).int(), offsets.int()


def _plain_product(s):
    c = s["case"]
    w = s["w"].detach()
    w = w.transpose(1, 2) if c["layout"] == "out_in" else w               # [experts, in, out]
    x = s["x"].detach()
    x = (x[s["order"].long() // c["top_k"]] if c["gather"] else x).float()
    rows = x.shape[0]
    y = torch.zeros(rows, c["out"], device=DEV)
    if c["train"]:
        g, dx, dw = s["g"].float(), torch.zeros(rows, c["in"], device=DEV), torch.zeros_like(w)
    # a product for each expert that has rows, as a program without such an operator has it
    for e, (a, b) in enumerate(zip(s["ends"], s["ends"][1:])):
        if a == b:
            continue
        we = w[e].float()
        torch.mm(x[a:b], we, out=y[a:b])
        if c["train"]:
            torch.mm(g[a:b], we.t(), out=dx[a:b])
            dw[e] = torch.mm(x[a:b].t(), g[a:b])
    y = y.to(s["x"].dtype)
    if not c["train"]:
        return y
    if c["gather"]:
        at = s["place"].view(-1, c["top_k"])
        dx = dx[at.long().clamp(min=0)].masked_fill(at[..., None] < 0, 0.0).sum(1)
    return y, dx.to(y.dtype), dw.transpose(1, 2) if c["layout"] == "out_in" else dw


def _plain_combine(s):
    c = s["case"]
    order, place, offsets = _order(s["at"], c["experts"])
    none = place < 0
    row = place.long().clamp(min=0)
    w = s["w"].detach().masked_fill(none, 0.0)
    y = s["y"].detach().float()[row].masked_fill(none[..., None], 0.0)    # [tokens, top_k, dim]
    out = (w[..., None] * y).sum(1).to(s["y"].dtype)
    if not c["train"]:
        return order, place, offsets, out
    g = s["g"].float()
    dw = (g[:, None] * y).sum(-1)
    token = order.long() // c["top_k"]
    dy = w.reshape(-1)[order.long(), None] * g[token]
    return order, place, offsets, out, dy.to(s["y"].dtype), dw


_PLAIN = {"append": _plain_append, "read": _plain_read, "attend": _plain_attend,
          "product": _plain_product, "combine": _plain_combine}


# ---------------------------------------------------- the framework's own ----
def _own_append(s):
    import paper_2608_06912_amd as L
    L.lapsum_cache_append(s["k_new"], s["v_new"], s["seen"], s["k"], s["v"], table=s["table"],
                          count=s["count"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return [s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None]


def _own_read(s):
    import paper_2608_06912_amd as L
    c = s["case"]
    return L.lapsum_cache_read(s["x"], s["lens"], c["len_max"], table=s["table"], scale=s["scale"],
                               dtype=getattr(torch, c["dtype"]))


def _own_attend(s):
    import paper_2608_06912_amd as L
    c = s["case"]
    out = L.lapsum_cache_attend(s["q"], s["k"], s["v"], s["lens"], table=s["table"],
                                k_scale=s["k_scale"], v_scale=s["v_scale"], window=c["window"],
                                lse=c["lse"], weights=c["weights"])
    return list(out) if c["lse"] or c["weights"] else [out]


def _own_product(s):
    import paper_2608_06912_amd.autograd as A
    c = s["case"]
    w = s["w"].transpose(1, 2) if c["layout"] == "out_in" else s["w"]
    gather = (s["order"], s["place"]) if c["gather"] else None
    y = A.expert_matmul(s["x"], w, s["offsets"], gather=gather)
    if not c["train"]:
        return y
    return (y.detach(), *torch.autograd.grad(y, (s["x"], s["w"]), s["g"]))


def _own_combine(s):
    import paper_2608_06912_amd as L
    import paper_2608_06912_amd.autograd as A
    c = s["case"]
    order, place, offsets = L.lapsum_expert_order(s["at"], c["experts"])
    out = A.expert_combine(s["y"], s["w"], place, offsets)
    if not c["train"]:
        return order, place, offsets, out
    return (order, place, offsets, out.detach(), *torch.autograd.grad(out, (s["y"], s["w"]), s["g"]))


_OWN = {"append": _own_append, "read": _own_read, "attend": _own_attend, "product": _own_product,
        "combine": _own_combine}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ------------------------------------------------------ floors and exact ----
_SIZE = {"float32": 4, "bfloat16": 2, "float16": 2, "int8": 1, "float8_e4m3fn": 1}


def work(c):
    """Inputs read once, outputs written once; of a cache only what the call
    concerns, of the matrices those of experts that have rows."""
    op = c["op"]
    if op in ("append", "read", "attend"):
        size = _SIZE[c["cache"]]
        row = c["dim"] * size + (4 if c["cache"] in MOST else 0)          # an entry of the cache
    if op == "append":
        m = 2 * c["kv"] * sum(_counts(c))
        return {"bytes": m * (row + c["dim"] * _SIZE[c["dtype"]]), "flops": 3 * m * c["dim"]}
    if op == "read":
        m, out = c["kv"] * sum(_lengths(c)), c["batch"] * c["kv"] * c["len_max"]
        return {"bytes": m * row + out * c["dim"] * _SIZE[c["dtype"]], "flops": m * c["dim"]}
    if op == "attend":
        live = sum(min(n, c["window"] or n) for n in _lengths(c))
        io = 2 * c["batch"] * c["heads"] * c["dim"] * _SIZE[c["dtype"]]
        room = -(-c["len_max"] // c["page"]) * c["page"] if c["paged"] else c["len_max"]
        more = 4 * c["batch"] * c["heads"] * room if c["weights"] else 0
        return {"bytes": 2 * c["kv"] * live * row + io + more, "flops": 4 * c["heads"] * live * c["dim"]}
    rows, size = c["tokens"] * c["top_k"], _SIZE[c["dtype"]]
    if op == "combine":
        more = (rows + c["tokens"]) * c["dim"] * size + 4 * rows if c["train"] else 0
        return {"bytes": (rows + c["tokens"]) * c["dim"] * size + 16 * rows + more,
                "flops": rows * c["dim"] * (6 if c["train"] else 2)}
    used = c["experts"] * (1.0 - (1.0 - 1.0 / c["experts"]) ** rows)
    ins = (c["tokens"] if c["gather"] else rows) * c["in"]
    weights = used * c["in"] * c["out"]
    rows_out = rows * c["out"]
    if c["train"]:   # rows, matrices and the gradient in; outputs and two gradients out
        return {"bytes": size * (2 * ins + weights + 2 * rows_out + c["experts"] * c["in"] * c["out"]),
                "flops": 6 * rows * c["in"] * c["out"]}
    return {"bytes": size * (ins + weights + rows_out), "flops": 2 * rows * c["in"] * c["out"]}


def _entry(s, n, b, p):
    """Where position p (a tensor) of sequence b is: (page, slot)."""
    if s["table"] is None:
        return torch.full_like(p, b), p
    size = s[n].shape[2]
    return s["table"][b].long()[p // size], p % size


def _live(s, n, b, p):
    """float64 [kv, positions, dim]: a cache's entries of sequence b."""
    page, slot = _entry(s, n, b, p)
    x = s[n].view(torch.int8) if s[n].dtype == torch.float8_e4m3fn else s[n]
    x = x[page, :, slot].view(s[n].dtype).double().transpose(0, 1)
    scale = s[n + "_scale"] if n != "x" else s["scale"]
    return x if scale is None else x * scale[page, :, slot].double().t()[..., None]


def _exact_append(s):
    c = s["case"]
    outs, scales = [], []
    for n in ("k", "v"):
        values = s[n].double() if c["cache"] != "int8" else None
        scale = s[n + "_scale"]
        scale = None if scale is None else scale.double()
        for b, count in enumerate(_counts(c)):
            p = c["seen"] + torch.arange(count, device=DEV)
            page, slot = _entry(s, n, b, p)
            x = s[n + "_new"][b, :, :count].double().transpose(0, 1)
            if scale is not None:
                unit = x.abs().amax(-1) / MOST[c["cache"]]
                scale[page, :, slot] = unit
                x = x / unit[..., None]
            if values is not None:
                values[page, :, slot] = x
        outs.append(values)
        scales += [] if scale is None else [scale]
    return outs + scales


def _exact_read(s):
    c = s["case"]
    out = torch.zeros(c["batch"], c["kv"], c["len_max"], c["dim"], dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(c)):
        out[b, :, :n] = _live(s, "x", b, torch.arange(n, device=DEV))
    return out


def _exact_attend(s):
    c = s["case"]
    group = c["heads"] // c["kv"]
    room = -(-c["len_max"] // c["page"]) * c["page"] if c["paged"] else c["len_max"]
    ys, lses, ws = [], [], []
    for b, n in enumerate(_lengths(c)):
        p = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device=DEV)
        k, v = _live(s, "k", b, p), _live(s, "v", b, p)
        q = s["q"][b].double().unflatten(0, (c["kv"], group))
        x = torch.stack([qh @ kh.t() for qh, kh in zip(q, k)]) / math.sqrt(c["dim"])
        w = torch.softmax(x, -1)
        ys.append(torch.cat([wh @ vh for wh, vh in zip(w, v)]))
        lses.append(torch.logsumexp(x, -1).reshape(-1))
        if c["weights"]:
            ws.append(torch.nn.functional.pad(w.flatten(0, 1), (int(p[0]), room - n)))
    out = [torch.stack(ys)]
    if c["lse"]:
        out.append(torch.stack(lses))
    if c["weights"]:
        out.append(torch.stack(ws))
    return out


def _exact_product(s):
    c = s["case"]
    w = s["w"].detach()
    x = s["x"].detach()
    rows = c["tokens"] * c["top_k"]
    y = torch.zeros(rows, c["out"], dtype=torch.float64, device=DEV)
    if c["train"]:
        dx, dw = torch.zeros(x.shape, dtype=torch.float64, device=DEV), torch.zeros(w.shape, dtype=torch.float64, device=DEV)
    at = s["offsets"].long()
    flat = s["order"].long()
    for e in range(c["experts"]):
        mine = torch.arange(int(at[e]), int(at[e + 1]), device=DEV)
        source = torch.div(flat[mine], c["top_k"], rounding_mode="floor") if c["gather"] else mine
        xe = x[source].double()
        we = w[e].double().t() if c["layout"] == "out_in" else w[e].double()
        y[mine] = xe @ we
        if c["train"]:
            ge = s["g"][mine].double()
            dx.index_add_(0, source, ge @ we.t())
            dw[e] = ge.t() @ xe if c["layout"] == "out_in" else xe.t() @ ge
    return (y, dx, dw) if c["train"] else y


def _exact_combine(s):
    c = s["case"]
    at = s["at"].reshape(-1)
    order = torch.cat([torch.nonzero(at == e)[:, 0] for e in range(c["experts"])])
    token = order // c["top_k"]
    w = s["w"].detach().double().reshape(-1)[order]
    y = s["y"].detach()[:order.numel()].double()
    out = torch.zeros(c["tokens"], c["dim"], dtype=torch.float64, device=DEV)
    out.index_add_(0, token, w[:, None] * y)
    if not c["train"]:
        return None, None, None, out
    g = s["g"].double()[token]
    dy = torch.zeros(at.numel(), c["dim"], dtype=torch.float64, device=DEV)
    dy[:order.numel()] = w[:, None] * g
    dw = torch.zeros(at.numel(), dtype=torch.float64, device=DEV)
    dw[order] = (g * y).sum(-1)
    return None, None, None, out, dy, dw.view(c["tokens"], c["top_k"])


_EXACT = {"append": _exact_append, "read": _exact_read, "attend": _exact_attend,
          "product": _exact_product, "combine": _exact_combine}


def exact(case, seed):
    return _EXACT[case["op"]](prepare(case, seed))
