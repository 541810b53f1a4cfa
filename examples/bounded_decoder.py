"""A small decoder that generates by beam search with a bounded key-value cache
and routed experts, the hard selections together as a model uses them:

  the prompt        attention over all of it; cache_accumulate over the weights of
                    its last queries, and cache_evict to the budget
  each new token    route_topk sends the rows to experts; cache_step adds up
                    the token's attention weights and gives it a slot
  each step         beam_select over beams and vocabulary, and beam_reorder of
                    every layer's keys, values, sums and positions

The model is random and tiny; what it computes besides is plain torch.

    python examples/bounded_decoder.py --budget 48 --new 24
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_06912_amd as L  # noqa: E402
import paper_2608_06912_amd.autograd as A  # noqa: E402


class Decoder:
    """layers x (attention with grouped heads, routed experts), learned positions."""

    def __init__(self, vocab=97, width=64, layers=2, heads=4, kv_heads=2, experts=8, chosen=2,
                 longest=512, seed=0, device="cuda", dtype=torch.float32):
        gen = torch.Generator(device="cpu").manual_seed(seed)
        self.heads, self.kv, self.dim, self.chosen = heads, kv_heads, width // heads, chosen

        def weight(*shape, scale=None):
            w = torch.randn(*shape, generator=gen) * (scale or shape[-2] ** -0.5)
            return w.to(device=device, dtype=dtype)

        self.embed, self.place = weight(vocab, width, scale=1.0), weight(longest, width, scale=0.5)
        self.out = weight(width, vocab, scale=2.0 * width ** -0.5)
        self.layers = [{
            "q": weight(width, heads * self.dim, scale=2.0 * width ** -0.5),
            "k": weight(width, kv_heads * self.dim), "v": weight(width, kv_heads * self.dim),
            "o": weight(heads * self.dim, width), "router": weight(width, experts),
            "bias": 0.05 * weight(1, experts, scale=1.0)[0].float(),
            "up": weight(experts, width, 2 * width), "down": weight(experts, 2 * width, width),
        } for _ in range(layers)]

    @staticmethod
    def norm(x):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    def project(self, layer, x):
        """q [rows, heads, tokens, dim], k and v [rows, kv_heads, tokens, dim]."""
        x = self.norm(x)
        return [(x @ layer[n]).unflatten(-1, (-1, self.dim)).transpose(1, 2).contiguous()
                for n in ("q", "k", "v")]

    def attend(self, q, k, v, mask):
        """Attention of grouped heads: (output [rows, tokens, heads dim], weights)."""
        group = self.heads // self.kv
        kk, vv = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        w = (q @ kk.transpose(2, 3).contiguous()) / math.sqrt(self.dim)
        w = torch.softmax(w.masked_fill(~mask, -math.inf), -1)
        return (w @ vv).transpose(1, 2).flatten(2), w

    def route(self, layer, logits):
        return A.route_topk(logits, self.chosen, score="sigmoid", bias=layer["bias"], groups=2,
                            topk_groups=1, group_top=2, renormalise=True)

    def experts(self, layer, x):
        """x plus its chosen experts' outputs."""
        h = self.norm(x).flatten(0, -2)
        weights, index = self.route(layer, h @ layer["router"])
        share = torch.zeros(h.shape[0], layer["up"].shape[0], device=h.device, dtype=h.dtype)
        share.scatter_(1, index.long(), weights.to(h.dtype))
        every = torch.relu(torch.stack([h @ up for up in layer["up"]]))
        every = torch.stack([y @ down for y, down in zip(every, layer["down"])], 1)
        return x + (share[..., None] * every).sum(1).view_as(x)

    def prompt(self, tokens, window):
        """Logits after the prompt [rows, tokens], and of each layer its keys,
        values and the last `window` queries' attention weights."""
        n = tokens.shape[1]
        x = self.embed[tokens] + self.place[:n]
        causal = torch.ones(n, n, dtype=torch.bool, device=x.device).tril()
        kept = []
        for layer in self.layers:
            q, k, v = self.project(layer, x)
            y, w = self.attend(q, k, v, causal)
            x = self.experts(layer, x + y @ layer["o"])
            kept.append((k, v, w[:, :, -window:]))
        return self.norm(x[:, -1]) @ self.out, kept

    def token(self, tokens, at, caches, insert):
        """Logits after one more token of each row, at position `at`; insert(layer
        number, cache, weights over its slots, k, v) puts its entry into the cache."""
        x = (self.embed[tokens] + self.place[at])[:, None]
        for i, (layer, cache) in enumerate(zip(self.layers, caches)):
            q, k, v = self.project(layer, x)
            there = cache["pos"].repeat_interleave(self.heads // self.kv, 1)[:, :, None] >= 0
            mask = torch.cat([there, torch.ones_like(there[..., :1])], -1)
            y, w = self.attend(q, torch.cat([cache["k"], k], 2), torch.cat([cache["v"], v], 2), mask)
            insert(i, cache, w[..., :-1], k, v)
            x = self.experts(layer, x + y @ layer["o"])
        return self.norm(x[:, 0]) @ self.out


def generate(model, prompt, new, beams=4, budget=64, window=8, sink=2, recent=16):
    """prompt [requests, tokens] -> (sequences [requests, beams, new], their
    scores), with caches of `budget` entries."""
    requests, length = prompt.shape
    logits, kept = model.prompt(prompt, window)
    seen = torch.full((requests,), length, dtype=torch.int32, device=prompt.device)
    caches = []
    for k, v, w in kept:
        acc = L.lapsum_cache_accumulate(w, model.kv, seen=seen)
        k, v, acc, pos = L.lapsum_cache_evict(k, v, acc, seen, budget, sink=sink, recent=recent)
        one = {"k": k, "v": v, "acc": acc, "pos": pos}
        caches.append({n: t.repeat_interleave(beams, 0) for n, t in one.items()})
    seen = seen.repeat_interleave(beams)

    def insert(i, cache, w, k, v):
        L.lapsum_cache_step(w, k, v, seen, cache["k"], cache["v"], cache["acc"], cache["pos"],
                            sink=sink, recent=recent)

    scores = torch.full((requests, beams), -math.inf, device=prompt.device)
    scores[:, 0] = 0.0                                  # one live beam before the first step
    logits = logits.repeat_interleave(beams, 0)
    chosen = torch.zeros(requests, beams, 0, dtype=torch.int64, device=prompt.device)
    for step in range(new):
        scores, tokens, parents = L.lapsum_beam_select(logits, scores, beams)
        if step:
            L.lapsum_beam_reorder([t for c in caches for t in c.values()], parents)
        take = parents.long()[..., None].expand(-1, -1, step)
        chosen = torch.cat([chosen.gather(1, take), tokens.long()[..., None]], -1)
        if step + 1 < new:
            logits = model.token(tokens.long().reshape(-1), length + step, caches, insert)
            seen += 1
    return chosen, scores


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=200)
    ap.add_argument("--new", type=int, default=24)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--budget", type=int, default=48)
    a = ap.parse_args()
    model = Decoder()
    gen = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randint(0, 97, (a.requests, a.prompt), generator=gen, device="cuda")
    for budget in (a.budget, a.prompt + a.new):
        chosen, scores = generate(model, prompt, a.new, a.beams, budget)
        print(f"{budget} cache entries:")
        for r in range(a.requests):
            print(f"  request {r}: {scores[r, 0].item():8.3f}  {chosen[r, 0].tolist()}")


if __name__ == "__main__":
    main()
