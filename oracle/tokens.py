"""A token and its confidence from a row of logits and one uniform number, in float64, from the
definition: rank the tokens, cut the list by count, by weight and by relative weight, draw from
what is left in index order."""
from __future__ import annotations

import math

import numpy as np


def sample_row(logits, temperature, top_k, top_p, min_p, u):
    """-> (token, confidence, kept tokens ascending, their weights).  Parameters as given, in
    float64; logits any float array, NaN as -inf."""
    l = np.asarray(logits, dtype=np.float64).copy()
    l[np.isnan(l)] = -np.inf
    if np.isposinf(l).any():
        l = np.where(np.isposinf(l), 0.0, -np.inf)
    m = l.max()
    if np.isneginf(m):
        return -1, 0.0, np.zeros(0, int), np.zeros(0)
    order = sorted(range(len(l)), key=lambda i: (-l[i], i)) if len(l) < 3000 else np.argsort(-l, kind="stable")
    order = np.asarray(order)
    flat = np.exp(l - m)
    if temperature == 0.0:
        token, kept, w = int(order[0]), order[:1], np.ones(1)
    else:
        w = np.exp((l[order] - m) / temperature)
        n = min(top_k, len(l)) if top_k > 0 else len(l)
        if top_p < 1.0:
            mass = math.fsum(w[:n])
            before, i = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]]), 0
            i = int((before < top_p * mass).sum())
            n = max(1, i)
        keep = w[:n] >= min_p
        keep[0] = True
        kept = order[:n][keep]
        kept = np.sort(kept[w[:n][keep] > 0.0])
        w = np.exp((l[kept] - m) / temperature)
        cum = np.cumsum(w)
        token = int(kept[min(int((cum <= u * cum[-1]).sum()), len(kept) - 1)])
    return token, float(flat[token] / flat.sum()), kept, w


def allowed(logits, temperature, top_k, top_p, min_p, u, slack):
    """The tokens that are right when shares of the weight are known to within `slack`."""
    out = set()
    for p in ({top_p} if top_p == 1.0 else {top_p, top_p * (1 - slack), min(1.0, top_p * (1 + slack))}):
        for q in {min_p, min_p * (1 - slack), min_p * (1 + slack)}:
            for v in (u, max(u - slack, 0.0), min(u + slack, 1.0 - 2.0 ** -53)):
                out.add(sample_row(logits, temperature, top_k, p, q, v)[0])
    return out
