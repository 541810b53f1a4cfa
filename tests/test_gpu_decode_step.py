"""A routed decoder that generates one token after another from a paged cache, the new
operators together as a model uses them: append, attend, route, order, the experts'
products and their sum.  Against the same model in float64 over whole sequences,
without a cache."""
import math

import pytest

pytestmark = pytest.mark.gpu


class Decoder:
    """layers x (attention with grouped heads, routed experts)."""

    def __init__(self, seed=0, vocab=61, width=64, layers=2, heads=4, kv=2, experts=6, chosen=2):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=gen, device="cuda") * s[-2] ** -0.5  # noqa: E731
        self.heads, self.kv, self.dim, self.chosen, self.experts = heads, kv, width // heads, chosen, experts
        self.embed, self.out = 8.0 * r(vocab, width), r(width, vocab)
        self.layers = [{"q": r(width, width), "k": r(width, kv * self.dim), "v": r(width, kv * self.dim),
                        "o": r(width, width), "router": 2.0 * r(width, experts), "up": r(experts, width, 2 * width),
                        "down": r(experts, 2 * width, width)} for _ in range(layers)]

    @staticmethod
    def norm(x):
        return x * (x * x).mean(-1, keepdim=True).add(1e-6).rsqrt()

    def step(self, tokens, seen, caches, table, lib, A):
        """Logits after one more token of each sequence; the caches take it in."""
        import torch
        x = self.embed[tokens]
        for layer, c in zip(self.layers, caches):
            h = self.norm(x)
            q, k, v = ((h @ layer[n]).unflatten(1, (-1, self.dim)) for n in "qkv")
            lib.lapsum_cache_append(k, v, seen, c["k"], c["v"], table=table, k_scale=c.get("ks"), v_scale=c.get("vs"))
            y = lib.lapsum_cache_attend(q, c["k"], c["v"], seen + 1, table=table, k_scale=c.get("ks"),
                                        v_scale=c.get("vs"))
            x = x + y.flatten(1) @ layer["o"]
            h = self.norm(x)
            w, at = A.route_topk(h @ layer["router"], self.chosen, renormalise=True)
            order, place, offsets = lib.lapsum_expert_order(at, self.experts)
            up = torch.relu(A.expert_matmul(h, layer["up"], offsets, gather=(order, place)))
            x = x + A.expert_combine(A.expert_matmul(up, layer["down"], offsets), w, place, offsets)
        return self.norm(x) @ self.out

    def whole(self, tokens):
        """float64 logits after every token of sequences [batch, n]."""
        import torch
        x = self.embed.double()[tokens]
        n = tokens.shape[1]
        causal = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for layer in self.layers:
            layer = {name: t.double() for name, t in layer.items()}
            h = self.norm(x)
            q, k, v = ((h @ layer[m]).unflatten(2, (-1, self.dim)).transpose(1, 2) for m in "qkv")
            k, v = (t.repeat_interleave(self.heads // self.kv, 1) for t in (k, v))
            s = (q[..., :, None, :] * k[..., None, :, :]).sum(-1) / math.sqrt(self.dim)
            a = torch.softmax(s.masked_fill(~causal, -math.inf), -1)
            y = (a[..., None] * v[..., None, :, :]).sum(-2)
            x = x + y.transpose(1, 2).flatten(2) @ layer["o"]
            h = self.norm(x)
            p = torch.softmax(h @ layer["router"], -1)
            top = p.topk(self.chosen, -1)
            share = torch.zeros_like(p).scatter(-1, top.indices, top.values / top.values.sum(-1, keepdim=True))
            every = torch.stack([torch.relu(h @ u) @ d for u, d in zip(layer["up"], layer["down"])], -2)
            x = x + (share[..., None] * every).sum(-2)
        return self.norm(x) @ self.out.double()


def _run(lib, kind, steps):
    import torch

    import paper_2608_06912_amd.autograd as A
    model = Decoder(seed=7)
    gen = torch.Generator(device="cuda").manual_seed(1)
    batch, slots, width = 3, 8, -(-steps // 8)
    pages = batch * width + 2
    table = torch.randperm(pages, generator=gen, device="cuda")[:batch * width].view(batch, width).int()
    tokens = torch.randint(0, 61, (batch, steps), generator=gen, device="cuda")
    caches = []
    for _ in model.layers:
        c = {n: torch.zeros(pages, model.kv, slots, model.dim, device="cuda").to(kind) for n in "kv"}
        if kind is not torch.float32:
            c |= {n: torch.ones(pages, model.kv, slots, device="cuda") for n in ("ks", "vs")}
        caches.append(c)
    seen = torch.zeros(batch, dtype=torch.int32, device="cuda")
    got = []
    for i in range(steps):
        got.append(model.step(tokens[:, i], seen, caches, table, lib, A))
        seen += 1
    return torch.stack(got, 1), model.whole(tokens)


def test_steps_are_the_whole_sequence(lib):
    import torch
    got, want = _run(lib, torch.float32, 21)
    assert float((got.double() - want).abs().max()) < 2e-3 * float(want.abs().max())


@pytest.mark.parametrize("kind,most", [("int8", 0.05), ("float8_e4m3fn", 0.25)])
def test_steps_from_a_cache_in_8_bits(lib, kind, most):
    """A code is off by half a step of its row's largest (int8: 1 / 254, e4m3: 1 / 16 of
    the value); the logits stay near in the mean."""
    import torch
    got, want = _run(lib, getattr(torch, kind), 21)
    assert float((got.double() - want).norm() / want.norm()) < most
