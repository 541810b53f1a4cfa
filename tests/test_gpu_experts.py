"""The experts' rows against plain float64: the order, the products and their
gradients, the weighted sum and its.

Tolerances count roundings: a sum of n products in float32 is off by at most
n 2^-24 of the sum of their magnitudes, and what is rounded to a type by half a
step of it, torch.finfo(t).eps / 2 of its value."""
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]


def _torch():
    import torch
    return torch


def _gen(seed):
    return _torch().Generator(device="cuda").manual_seed(seed)


def _close(got, want, size, n, dtype=None):
    """got is want up to n float32 roundings of `size` and one to its type."""
    torch = _torch()
    half = torch.finfo(dtype or got.dtype).eps / 2
    room = n * 2.0 ** -24 * size + half * (want.abs() + n * 2.0 ** -24 * size) + 2.0 ** -140
    if (dtype or got.dtype) is torch.float16:   # its steps stop at 2^-24
        room = room + 2.0 ** -25
    off = (got.double() - want).abs()
    assert got.shape == want.shape and bool((off <= room).all()), float((off / room).max())


def _indices(tokens, top_k, experts, seed, none=0.1, kind="spread"):
    torch = _torch()
    gen = _gen(seed)
    at = torch.randint(0, experts, (tokens, top_k), generator=gen, device="cuda", dtype=torch.int32)
    if kind == "one":
        at.fill_(experts - 1)
    elif kind == "skew":
        at = torch.where(torch.rand(at.shape, generator=gen, device="cuda") < 0.7, 0, at).int()
    gone = torch.rand(at.shape, generator=gen, device="cuda")
    at[gone < none] = -1
    at[gone < none / 2] = experts + 3
    return at


def _order_of(at, experts):
    torch = _torch()
    key = torch.where((at >= 0) & (at < experts), at, experts).reshape(-1).cpu()
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(key.numel())
    place[key == experts] = -1
    offsets = torch.tensor([int((key < e).sum()) for e in range(experts + 1)], dtype=torch.int32)
    return order.int(), place.view(at.shape).int(), offsets


@pytest.mark.parametrize("tokens,top_k,experts,kind", [
    (0, 2, 5, "spread"), (1, 1, 1, "spread"), (1, 4, 64, "spread"), (63, 1, 2, "spread"), (16, 4, 63, "spread"),
    (1024, 8, 64, "one"), (1025, 8, 64, "skew"), (4096, 2, 1, "spread"), (8193, 1, 2048, "spread"),
    (40003, 3, 37, "skew"), (30000, 8, 256, "spread"), (70001, 2, 511, "one")])
def test_order(lib, tokens, top_k, experts, kind):
    at = _indices(tokens, top_k, experts, tokens + experts, kind=kind)
    for got, want in zip(lib.lapsum_expert_order(at, experts), _order_of(at, experts)):
        assert got.shape == want.shape and bool((got.cpu() == want).all())


SHAPES = [  # tokens, top_k, experts, in, out
    (1, 1, 1, 1, 1), (3, 2, 4, 8, 8), (5, 1, 3, 33, 7), (16, 4, 64, 256, 136), (130, 2, 5, 64, 128),
    (257, 3, 7, 100, 260), (64, 2, 200, 40, 24), (300, 1, 1, 129, 131), (700, 2, 3, 192, 320),
]


def _weights(experts, n_in, n_out, layout, dtype, gen):
    torch = _torch()
    if layout == "out_in":
        return torch.randn(experts, n_out, n_in, generator=gen, device="cuda").to(dtype).transpose(1, 2)
    return torch.randn(experts, n_in, n_out, generator=gen, device="cuda").to(dtype)


def _by_expert(rows, offsets):
    ends = offsets.tolist()
    return [(e, a, b) for e, (a, b) in enumerate(zip(ends, ends[1:])) if a < b]


# those of the largest tiles, of gradients in tiles of each size, and of both ways to LDS
LARGE = [(8200, 2, 3, 2600, 2056), (8200, 2, 3, 1504, 2056), (8200, 2, 3, 72, 2056), (8200, 2, 3, 1501, 2055)]


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", LARGE)
def test_large_products_and_their_gradients(lib, shape, dtype, layout):
    _products(lib, shape, dtype, layout, True)


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_products_and_their_gradients(lib, shape, dtype, layout, gather):
    _products(lib, shape, dtype, layout, gather)


def _products(lib, shape, dtype, layout, gather):
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    tokens, top_k, experts, n_in, n_out = shape
    dtype = getattr(torch, dtype)
    gen = _gen(sum(shape))
    order, place, offsets = lib.lapsum_expert_order(_indices(tokens, top_k, experts, 7 + tokens), experts)
    rows = tokens * top_k
    x = torch.randn(tokens if gather else rows, n_in, generator=gen, device="cuda").to(dtype)
    w = _weights(experts, n_in, n_out, layout, dtype, gen)
    g = torch.randn(rows, n_out, generator=gen, device="cuda").to(dtype)
    x.requires_grad_()
    w.requires_grad_()
    y = A.expert_matmul(x, w, offsets, gather=(order, place) if gather else None)
    dx, dw = torch.autograd.grad(y, (x, w), g)
    assert dw.stride() == w.stride() or experts == 1 or 1 in w.shape
    xs, ws, gs = x.detach().double(), w.detach().double(), g.double()
    if gather:
        xs = xs[order.long() // top_k]
    want = {n: torch.zeros(s, dtype=torch.float64, device="cuda") for n, s in
            (("y", (rows, n_out)), ("dx", (rows, n_in)), ("dw", w.shape))}
    size = {n: torch.zeros_like(t) for n, t in want.items()}
    for e, a, b in _by_expert(rows, offsets):
        for out, f in ((want, lambda t: t), (size, torch.abs)):
            out["y"][a:b] = f(xs[a:b]) @ f(ws[e])
            out["dx"][a:b] = f(gs[a:b]) @ f(ws[e]).t().contiguous()
            out["dw"][e] = f(xs[a:b]).t().contiguous() @ f(gs[a:b])
    if gather:
        token = order.long() // top_k
        for out in (want, size):
            out["dx"] = torch.zeros(tokens, n_in, dtype=torch.float64, device="cuda").index_add_(0, token, out["dx"])
    _close(y.detach(), want["y"], size["y"], n_in)
    _close(dx, want["dx"], size["dx"], n_out + top_k)
    _close(dw, want["dw"], size["dw"], rows)
    end = int(offsets[-1])
    assert not y[end:].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_products_read_views_and_leave_what_is_beside_them(lib, dtype):
    """Rows with a stride, at odd addresses, matrices cut out of larger ones; NaN all around."""
    torch = _torch()
    dtype = getattr(torch, dtype)
    gen = _gen(3)
    order, place, offsets = lib.lapsum_expert_order(_indices(50, 2, 4, 5, none=0.0), 4)
    big = torch.full((52, 40), float("nan"), device="cuda", dtype=dtype)
    x = big[1:51, 3:36]
    x.copy_(torch.randn(50, 33, generator=gen, device="cuda"))
    wide = torch.full((4, 35, 61), float("nan"), device="cuda", dtype=dtype)
    w = wide[:, 1:34, 2:57]
    w.copy_(torch.randn(4, 33, 55, generator=gen, device="cuda"))
    for a, b in ((x, w), (x.contiguous(), w.contiguous())):
        y = lib.lapsum_expert_matmul(a, b, offsets, order=order, top_k=2)
        want = torch.cat([x[order.long() // 2][i:j].double() @ w[e].double() for e, i, j in _by_expert(100, offsets)])
        _close(y, want, 33 * 25.0, 33)


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", TYPES)
def test_lines_of_every_short_length(lib, dtype, layout):
    """A line's last chunk, whole, in part and shorter than a vector, NaN on both sides of it; values whose sums
    are exact in every type (at most 4 x 23), so that results are equal."""
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    dtype = getattr(torch, dtype)
    gen = _gen(11)
    offsets = torch.tensor([0, 6, 6, 23], dtype=torch.int32, device="cuda")

    def cut(*shape):
        big = torch.full((*shape[:-1], shape[-1] + 2), float("nan"), device="cuda", dtype=dtype)
        view = big[..., 1:-1]
        view.copy_(torch.randint(-2, 3, shape, generator=gen, device=gen.device))
        return view

    for n_in in range(1, 20):
        for n_out in (1, 2, 3, 5, 7, 9, 12, 15, 17, 19):
            x = cut(23, n_in).requires_grad_()
            w = cut(3, n_in, n_out) if layout == "in_out" else cut(3, n_out, n_in).transpose(1, 2)
            w.requires_grad_()
            g = cut(23, n_out)
            y = A.expert_matmul(x, w, offsets)
            dx, dw = torch.autograd.grad(y, (x, w), g)
            xd, wd, gd = (t.detach().double().cpu() for t in (x, w, g))
            for e, (lo, hi) in enumerate(((0, 6), (6, 6), (6, 23))):
                case = (n_in, n_out, e)
                assert torch.equal(y[lo:hi].detach().double().cpu(), xd[lo:hi] @ wd[e]), case
                assert torch.equal(dx[lo:hi].double().cpu(), gd[lo:hi] @ wd[e].T), case
                assert torch.equal(dw[e].double().cpu(), xd[lo:hi].T @ gd[lo:hi]), case


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,n_in,n_out", [
    (40, 8, 64, 77), (500, 3, 40, 131), (8192, 4, 64, 1021), (8192, 1, 64, 4041), (8192, 1, 64, 4044)])
def test_whole_vectors_in_and_odd_rows_out(lib, rows, experts, n_in, n_out, dtype):
    """Matrices stored [out, in]: what is read is in whole vectors, what is written not.  Sums of at most 64
    products of at most 4 are exact in every type, so that results are equal."""
    torch = _torch()
    dtype = getattr(torch, dtype)
    gen = _gen(12)
    draw = lambda *s: torch.randint(-2, 3, s, generator=gen, device=gen.device).cuda().to(dtype)  # noqa: E731
    x, w = draw(rows, n_in), draw(experts, n_out, n_in).transpose(1, 2)
    ends = torch.linspace(0, rows - 5, experts + 1).int().cuda()
    y = lib.lapsum_expert_matmul(x, w, ends)
    for e, lo, hi in _by_expert(rows, ends):
        assert torch.equal(y[lo:hi].double(), x[lo:hi].double() @ w[e].double()), e
    assert not bool(y[rows - 5:].any())


def test_rows_without_an_expert_may_hold_anything(lib):
    torch = _torch()
    x = torch.randn(6, 16, device="cuda")
    x[4:] = float("nan")
    offsets = torch.tensor([0, 1, 1, 4], dtype=torch.int32, device="cuda")
    w = torch.randn(3, 16, 8, device="cuda")
    w[1] = float("inf")
    y = lib.lapsum_expert_matmul(x, w, offsets)
    assert bool(torch.isfinite(y).all()) and not y[4:].any() and bool(y[:4].any(1).all())
    dw = lib.lapsum_expert_matmul_weights(x, torch.randn(6, 8, device="cuda"), offsets, w)
    assert bool(torch.isfinite(dw).all()) and not dw[1].any()


def test_offsets_and_orders_that_lie_stay_inside(lib):
    """Offsets out of range or falling, and orders of rows that are none: no access outside."""
    torch = _torch()
    x, w = torch.randn(40, 24, device="cuda"), torch.randn(3, 24, 16, device="cuda")
    for ends in ([0, 50, 7, 90], [-5, 10, 20, 1 << 30], [40, 30, 20, 10]):
        offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        assert lib.lapsum_expert_matmul(x, w, offsets).shape == (40, 16)
        assert lib.lapsum_expert_matmul_weights(x, torch.randn(40, 16, device="cuda"), offsets, w).shape == w.shape
    order = torch.tensor([0, 79, 80, -1, 1 << 30], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 5, 5, 5], dtype=torch.int32, device="cuda")
    y = lib.lapsum_expert_matmul(x, w, offsets, order=order, top_k=2)
    assert bool(y[:2].any(1).all()) and not y[2:].any()
    place = torch.tensor([[0, 39], [-1, 40], [1 << 30, 3]], dtype=torch.int32, device="cuda")
    out = lib.lapsum_expert_combine(x, place)
    assert bool(torch.equal(out, torch.stack([x[0] + x[39], 0 * x[0], x[3]])))


def test_gradients_are_those_of_differences(lib):
    """The products are linear in each of their inputs, so a central difference is exact up
    to its roundings: two values of about 1e2 to 2^-22, over a step of 2."""
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    gen = _gen(9)
    order, place, offsets = lib.lapsum_expert_order(_indices(12, 2, 3, 1), 3)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, w, p = r(12, 10), r(3, 10, 6), torch.rand(12, 2, generator=gen, device="cuda")
    g = r(12, 6)

    def f(x, w, p):
        y = A.expert_matmul(x, w, offsets, gather=(order, place))
        return A.expert_combine(y, p, place, offsets)

    leaves = [t.clone().requires_grad_() for t in (x, w, p)]
    grads = torch.autograd.grad(f(*leaves), leaves, g)
    for n in range(3):
        d = r(*leaves[n].shape)
        args = [[t + s * d if i == n else t for i, t in enumerate((x, w, p))] for s in (1.0, -1.0)]
        up, down = (f(*a).double() for a in args)
        slope = ((up - down) * g.double()).sum() / 2
        assert abs(float(slope - (grads[n].double() * d.double()).sum())) < 1e-3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,top_k,experts,dim", [
    (0, 2, 3, 8), (1, 1, 1, 1), (5, 3, 4, 7), (16, 4, 64, 2048), (33, 8, 16, 520), (100, 2, 5, 1001),
    (9, 64, 100, 264), (20, 2, 6, 4104)])
def test_weighted_sum_and_its_gradients(lib, tokens, top_k, experts, dim, dtype):
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    dtype = getattr(torch, dtype)
    gen = _gen(tokens + dim)
    order, place, offsets = lib.lapsum_expert_order(_indices(tokens, top_k, experts, 11 + dim), experts)
    y = torch.randn(tokens * top_k, dim, generator=gen, device="cuda").to(dtype).requires_grad_()
    p = torch.randn(tokens, top_k, generator=gen, device="cuda").requires_grad_()
    g = torch.randn(tokens, dim, generator=gen, device="cuda").to(dtype)
    out = A.expert_combine(y, p, place, offsets)
    dy, dp = torch.autograd.grad(out, (y, p), g)
    here = (place >= 0)[..., None]
    ys = torch.where(here, y.detach().double()[place.long().clamp(min=0)], 0.0) if tokens else \
        torch.zeros(0, top_k, dim, dtype=torch.float64, device="cuda")
    ps, gs = p.detach().double()[..., None], g.double()[:, None]
    _close(out.detach(), (ps * ys).sum(1), (ps * ys).abs().sum(1), top_k + 1)
    _close(dp, (gs * ys).sum(-1), (gs * ys).abs().sum(-1), dim + 1)
    want = torch.zeros(tokens * top_k, dim, dtype=torch.float64, device="cuda")
    want[place[place >= 0].long()] = torch.where(here, ps * gs, 0.0)[place >= 0]
    _close(dy, want, want.abs(), 1)
    if dtype is torch.float32 and tokens:   # without weights, into another type
        half = lib.lapsum_expert_combine(y.detach(), place, dtype=torch.bfloat16)
        _close(half, ys.sum(1), ys.abs().sum(1), top_k)


def test_a_routed_layer_as_a_whole(lib):
    """route_topk, the order, two products and the sum, against float64 and its autograd."""
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    gen = _gen(21)
    tokens, experts, k, width, inner = 70, 6, 2, 48, 72
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    leaves = [r(tokens, experts), r(tokens, width), r(experts, width, inner) / 7, r(experts, inner, width) / 8]
    g = r(tokens, width)
    logits, x, up, down = [t.clone().requires_grad_() for t in leaves]
    p, at = A.route_topk(logits, k, score="softmax", renormalise=True)
    order, place, offsets = lib.lapsum_expert_order(at, experts)
    h = torch.relu(A.expert_matmul(x, up, offsets, gather=(order, place)))
    out = A.expert_combine(A.expert_matmul(h, down, offsets), p, place, offsets)
    grads = torch.autograd.grad(out, (logits, x, up, down), g)
    logits, x, up, down = [t.double().requires_grad_() for t in leaves]
    s = torch.softmax(logits, -1).gather(1, at.long())
    s = s / s.sum(-1, keepdim=True)
    every = torch.stack([torch.relu(x @ up[e]) @ down[e] for e in range(experts)], 1)
    want = (s[..., None] * every.gather(1, at.long()[..., None].expand(-1, -1, width))).sum(1)
    wants = torch.autograd.grad(want, (logits, x, up, down), g.double())
    # sums of at most 140 products of normal numbers after sums of 72: 2^-24 (140 + 72) of
    # magnitudes below 64
    for a, b in zip((out, *grads), (want, *wants)):
        assert float((a.double() - b).detach().abs().max()) < 64 * 212 * 2.0 ** -24


def test_what_is_not_a_gradient_is_refused(lib):
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    order, place, offsets = lib.lapsum_expert_order(_indices(4, 2, 3, 2), 3)
    x, w = torch.randn(4, 8, device="cuda", requires_grad=True), torch.randn(3, 8, 8, device="cuda")
    y = A.expert_matmul(x, w, offsets, gather=(order, place))
    (dx,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dx.sum(), x)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(x.detach(), torch.ones_like(x))
        with pytest.raises(RuntimeError):
            A.expert_matmul(dual, w, offsets, gather=(order, place))
    for bad in (dict(w=w.half()), dict(w=w[:, :7]), dict(offsets=offsets[:3]), dict(offsets=offsets.long()),
                dict(w=w.cpu()), dict(x=x[0]), dict(gather=(order, place[:, :1])), dict(x=x.double())):
        kw = {"x": x, "w": w, "offsets": offsets, "gather": (order, place), **bad}
        with pytest.raises((ValueError, RuntimeError)):
            A.expert_matmul(kw["x"], kw["w"], kw["offsets"], gather=kw["gather"])
    with pytest.raises(lib.LapsumError):
        lib.lapsum_expert_order(place, 0)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_expert_order(place, 2049)
    with pytest.raises(ValueError):
        lib.lapsum_expert_order(place.long(), 3)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_expert_matmul(x.detach(), w, offsets, order=order, top_k=0)


def test_captured_and_replayed(lib):
    """A layer's forward and backward as a graph, replayed on new inputs with eager work
    between: each replay as the eager call."""
    import paper_2608_06912_amd.autograd as A
    torch = _torch()
    gen = _gen(33)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    tokens, experts, k = 90, 5, 2
    at, x, w, p, g = (_indices(tokens, k, experts, 1), r(tokens, 64), r(experts, 64, 40), r(tokens, k), r(tokens, 40))

    def step():
        a, b, c = (t.detach().requires_grad_() for t in (x, w, p))
        order, place, offsets = lib.lapsum_expert_order(at, experts)
        out = A.expert_combine(A.expert_matmul(a, b, offsets, gather=(order, place)), c, place, offsets)
        return (out.detach(), *torch.autograd.grad(out, (a, b, c), g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(4):
        at.copy_(_indices(tokens, k, experts, 50 + turn, kind=["spread", "one", "skew", "spread"][turn]))
        x.copy_(r(tokens, 64))
        g.copy_(r(tokens, 40))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step()):
            assert bool(torch.equal(a, b))


def test_on_another_stream(lib):
    torch = _torch()
    order, place, offsets = lib.lapsum_expert_order(_indices(300, 2, 8, 4), 8)
    x, w = torch.randn(300, 128, device="cuda").half(), torch.randn(8, 128, 256, device="cuda").half()
    want = lib.lapsum_expert_matmul(x, w, offsets, order=order, top_k=2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        x2 = x * 2
        got = lib.lapsum_expert_matmul(x2, w, offsets, order=order, top_k=2)
    side.synchronize()
    assert bool(torch.equal(got, want * 2))
