"""Float64 oracle of the hard selections (NumPy only; it shares no code with the
library): routing to experts and its gradient, a beam search's step, a cache
cut to a budget and its single-token step, each from its definition.

Larger values first, equal ones by the lowest index; NaN never before a
number.  `value` results are what a selection compares, in float64, so that a test can
allow for values that differ by less than float32 holds.
"""
from __future__ import annotations

import numpy as np


def best(value, k):
    """Indices of the k largest of a vector that are neither NaN nor -inf,
    larger first, equal ones by the lowest index."""
    v = np.where(np.isnan(value), -np.inf, value)
    order = np.lexsort((np.arange(v.size), -v))
    return [int(i) for i in order[:k] if v[i] > -np.inf]


# -------------------------------------------------------------- routing ----
def clean_logits(x):
    """Logits as the definition takes them: NaN masked, +inf the largest float."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    return np.minimum(x, float(np.finfo(np.float32).max))


def route_scores(x, score):
    """s of one token."""
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-x))
    top = x.max()
    if top == -np.inf:
        return np.zeros_like(x)
    e = np.exp(x - top)
    return e / e.sum()


def route_values(x, score, bias=None, groups=1, topk_groups=None, group_top=1):
    """(c of the experts that may be chosen, -inf elsewhere) of one token."""
    s = route_scores(x, score)
    if score == "softmax" and bias is None:
        c = x.copy()
        top = x.max()
        by_group = c if group_top == 1 or top == -np.inf else \
            np.where(x > -np.inf, np.exp(x - top), -np.inf)
    else:
        c = s if bias is None else s + bias
        c = np.where(x == -np.inf, -np.inf, np.where(np.isnan(c), -np.inf, c))
        by_group = c
    topk_groups = groups if topk_groups is None else topk_groups
    if topk_groups < groups:
        parts = by_group.reshape(groups, -1)
        g = np.full(groups, -np.inf)
        for j in range(groups):
            b = sorted(parts[j], reverse=True)[:group_top]
            b = [v for v in b if v > -np.inf]
            if b:
                g[j] = sum(b)
        order = np.lexsort((np.arange(groups), -g))[:topk_groups]
        kept = np.zeros(groups, bool)
        kept[order] = True
        c = np.where(np.repeat(kept, c.size // groups), c, -np.inf)
    return c


def route_weights(x, chosen, score, renormalise, scale):
    """Weights of the chosen experts (a list of indices) of one token."""
    if not chosen:
        return np.zeros(0)
    if renormalise and score == "softmax":
        e = np.exp(x[chosen] - x[chosen].max())
        return scale * e / e.sum()
    s = route_scores(x, score)[chosen]
    if not renormalise:
        return scale * s
    return scale * s / s.sum() if s.sum() > 0 else 0.0 * s


def route_gradient(x, chosen, g, score, renormalise, scale):
    """dL/dx of one token for dL/dw = g over the chosen experts, from the
    derivative of each weight with respect to each logit."""
    n = x.size
    if not chosen:
        return np.zeros(n)
    idx = np.asarray(chosen)
    g = np.asarray(g, np.float64)
    s = route_scores(x, score)
    if score == "sigmoid":
        t = np.exp(-np.abs(x))
        ds = np.diag(t / (1.0 + t) ** 2)[idx]          # [chosen, n]
    else:
        ds = np.diag(s)[idx] - np.outer(s[idx], s)
    if renormalise:
        total = s[idx].sum()
        if total == 0.0:
            return np.zeros(n)
        ds = ds / total - np.outer(s[idx], ds.sum(0)) / total ** 2
    return scale * (g @ ds)


# ---------------------------------------------------------- beam search ----
def beam_scores(logits, cum):
    """s of every continuation of one request, float64 [beams, vocab]."""
    x = np.asarray(logits, np.float64)
    out = np.full(x.shape, np.nan)
    for w in range(x.shape[0]):
        top = np.max(x[w])
        if not np.isfinite(top):
            continue                                   # NaN, +inf, or nothing
        out[w] = float(cum[w]) + (x[w] - (top + np.log(np.exp(x[w] - top).sum())))
    return out


# ---------------------------------------------------------------- cache ----
def accumulate(weights, kv, seen=None, acc=None):
    w = np.asarray(weights, np.float64)
    batch, heads, queries, keys = w.shape
    w = w.reshape(batch, kv, heads // kv * queries, keys)
    out = np.zeros((batch, kv, keys)) if acc is None else np.asarray(acc, np.float64).copy()
    for b in range(batch):
        n = keys if seen is None else max(0, min(int(seen[b]), keys))
        out[b, :, :n] += w[b, :, :, :n].sum(1)
    return out


def kept_slots(acc, pos, seen, budget, sink, recent):
    """Slots of one (sequence, head) that stay, ascending."""
    live = pos >= 0
    always = live & ((pos < sink) | (pos >= max(0, seen - recent)))
    none = np.isnan(acc) & ~always
    value = np.where(always | none, 0.0, acc)
    order = np.lexsort((np.arange(acc.size), -value, none, ~always, ~live))
    return sorted(int(i) for i in order[:min(budget, int(live.sum()))])


def step_slot(acc, pos, now, sink, recent):
    """The slot that a new token at position `now` takes."""
    empty = np.nonzero(pos < 0)[0]
    if empty.size:
        return int(empty[0])
    free = (pos >= sink) & (pos < now - recent + 1)
    at = np.nonzero(free)[0]
    if not at.size:
        return 0
    nan = at[np.isnan(acc[at])]
    if nan.size:
        return int(nan[0])
    return int(at[np.argmin(acc[at])])
