"""The matrix product over rows with its epilogue, and sampling, from their definitions in fp64.  No code is shared with the
library."""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def activate(v, act):
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "relu":
            return np.where(v < 0, 0.0, v)
        if act == "gelu":
            return 0.5 * v * (1.0 + _erf(v / math.sqrt(2.0)))
        if act == "gelu_tanh":
            return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        if act == "silu":
            return v / (1.0 + np.exp(-v))
    assert act == "none"
    return v


def linear(x, w, bias=None, residual=None, act="none", mode="none"):
    """(y, s, size): the result, the sums before the activation and the sum of the absolute terms, all fp64."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        s, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        s, size = s + np.asarray(bias, dtype=np.float64), size + np.abs(np.asarray(bias, dtype=np.float64))
    if mode == "before":
        s, size = s + residual, size + np.abs(residual)
    y = activate(s, act)
    if mode == "after":
        y, size = y + residual, size + np.abs(residual)
    return y, s, size


def sample_row(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, probs) of one row, by sorting the candidates."""
    l = np.asarray(l, dtype=np.float64)
    probs = np.zeros(len(l))
    cand = np.flatnonzero(l > -np.inf)                     # a NaN compares false
    if len(cand) == 0:
        return -1, 0.0, probs
    order = cand[np.lexsort((cand, -l[cand]))]
    top = l[order[0]]
    if np.isinf(top):
        order = order[l[order] == top]
    if not temperature > 0.0:
        order = order[:1]
    if top_k > 0:
        order = order[:top_k]
    w = np.ones(len(order)) if np.isinf(top) or not temperature > 0.0 else np.exp((l[order] - top) / temperature)
    if top_p < 1.0:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        stay = before < top_p * np.sum(w)
        stay[0] = True
        order, w = order[stay], w[stay]
    if min_p > 0.0:
        stay = w >= min(min_p, 1.0)
        order, w = order[stay], w[stay]
    at = np.argsort(order)
    order, w = order[at], w[at]
    mass = np.cumsum(w)
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    i = min(int(np.searchsorted(mass, u * mass[-1], side="right")), len(order) - 1)
    probs[order] = w / mass[-1]
    return int(order[i]), float(probs[order[i]]), probs
