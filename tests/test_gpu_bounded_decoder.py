"""The example decoder with room for every entry against the same model without
any cache, in float64 and plain torch; and with a budget, what its caches hold."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _plain(model, prompt, new, beams, D):
    """Beam search that runs the model over every sequence from its start."""
    import torch

    class Plain(D.Decoder):
        def __init__(self, of):
            self.heads, self.kv, self.dim, self.chosen = of.heads, of.kv, of.dim, of.chosen
            self.embed, self.place, self.out = of.embed.double(), of.place.double(), of.out.double()
            self.layers = [{n: w.double() for n, w in layer.items()} for layer in of.layers]

        def route(self, layer, logits):
            s = torch.sigmoid(logits)
            c = (s + layer["bias"]).view(s.shape[0], 2, -1)
            first = c.topk(2).values.sum(-1).argmax(-1)
            out = torch.arange(2, device=s.device) != first[:, None]
            at = c.masked_fill(out[..., None], -math.inf).flatten(1).topk(self.chosen).indices
            w = s.gather(1, at)
            return w / w.sum(-1, keepdim=True), at

    plain = Plain(model)
    rows, best = prompt.shape[0], []
    for r in range(rows):
        live = [(0.0, [])]
        for _ in range(new):
            seqs = torch.tensor([prompt[r].tolist() + s for _, s in live], device=prompt.device)
            logp = torch.log_softmax(plain.prompt(seqs, 1)[0], -1).tolist()
            every = [(sc + lp, s + [v]) for (sc, s), row in zip(live, logp) for v, lp in enumerate(row)]
            live = sorted(every, key=lambda e: -e[0])[:beams]
        best.append(live)
    return best


def test_with_room_for_all_it_is_the_plain_model(lib):
    import torch

    import bounded_decoder as D
    model = D.Decoder(vocab=41, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(5)
    prompt = torch.randint(0, 41, (2, 19), generator=gen, device="cuda")
    chosen, scores = D.generate(model, prompt, 6, beams=3, budget=40)
    for r, live in enumerate(_plain(model, prompt, 6, 3, D)):
        assert chosen[r].tolist() == [s for _, s in live]
        for b, (score, _) in enumerate(live):
            assert abs(float(scores[r, b]) - score) < 1e-3


def test_a_budget_bounds_the_caches_and_keeps_the_ends(lib, monkeypatch):
    import torch

    import bounded_decoder as D
    model = D.Decoder(seed=4)
    prompt = torch.randint(0, 97, (2, 120), device="cuda")
    caches = []
    step = D.L.lapsum_cache_step

    def watch(*args, **kw):
        slot = step(*args, **kw)
        caches[:] = [args[7]]
        assert kw == {"sink": 2, "recent": 16}
        pos, now = args[7], int(args[3][0])
        assert pos.shape[-1] == 32 and bool((pos >= 0).all())
        for p in pos.flatten(0, 1).tolist():
            assert len(set(p)) == 32 and {0, 1} <= set(p) and set(range(now - 15, now + 1)) <= set(p)
        return slot

    monkeypatch.setattr(D.L, "lapsum_cache_step", watch)
    chosen, scores = D.generate(model, prompt, 30, beams=4, budget=32)
    assert caches and chosen.shape == (2, 4, 30) and bool(torch.isfinite(scores).all())
    assert bool((scores[:, :-1] >= scores[:, 1:]).all())
