"""From hidden states to the next tokens -- CPU oracle, TEST INFRASTRUCTURE ONLY.

Products with 8-bit weights, rules on the logits and the draw of a token, from their definitions: numpy,
fp64, with fp32 where a definition names it (what decides a code is decided in the stated type).
"""
from __future__ import annotations

import numpy as np

F = np.float32


def quantise(x: np.ndarray, floor: float):
    """Codes and step of a row of fp32 values."""
    if not np.isfinite(x).all():
        return np.zeros(x.shape, np.int64), F(np.nan)
    a = max(F(np.abs(x).max()), F(floor))
    return np.rint(x * (F(127.0) * (F(1.0) / a))).astype(np.int64), a / F(127.0)


def linear(x: np.ndarray, codes: np.ndarray, steps: np.ndarray) -> np.ndarray:
    """x [M, K] fp32 values, codes [N, K] integers, steps [N]: fp64 [M, N], integer sums exact."""
    out = np.empty((len(x), len(codes)))
    for m, row in enumerate(x):
        q, d = quantise(row, 1e-5)
        out[m] = (codes.astype(np.int64) @ q) * float(d) * steps.astype(np.float64)
    return out


def adjust(x, history=None, start=0, repetition=1.0, presence=0.0, frequency=0.0, bias=None, allowed=None):
    """One row: x fp32 [V], history the tokens that count, bias [V], allowed bool [V]; fp32 operations."""
    x = x.astype(F).copy()
    V = len(x)
    if history is not None:
        h = np.asarray(history)
        seen = np.zeros(V, bool)
        seen[h[(h >= 0) & (h < V)]] = True
        made = np.asarray(h[start:])
        count = np.bincount(made[(made >= 0) & (made < V)], minlength=V)
        with np.errstate(all="ignore"):
            x = np.where(seen, np.where(x > 0, x / F(repetition), x * F(repetition)), x)
            x = np.where(count > 0, x - count.astype(F) * F(frequency) - F(presence), x)
    if bias is not None:
        with np.errstate(invalid="ignore"):
            x = x + bias.astype(F)
    if allowed is not None:
        x = np.where(allowed, x, F(-np.inf))
    return x.astype(F)


def kept(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: the kept tokens in the row's order, every token's weight (fp64), and how far the nearest
    undecided weight sum is from top_p's border, relative to the sum."""
    x = np.minimum(np.where(np.isnan(x), -np.inf, x.astype(np.float64)), float(np.finfo(F).max))
    top = x.max()
    if top == -np.inf:
        return np.zeros(0, np.int64), np.zeros(len(x)), 1.0
    order = np.lexsort((np.arange(len(x)), -x))
    if temperature == 0:
        w = np.zeros(len(x))
        w[order[0]] = 1.0
        return order[:1], w, 1.0
    with np.errstate(under="ignore"):
        w = np.exp((x - top) / float(temperature))
    n = len(x) if top_k <= 0 else min(len(x), top_k)
    if min_p > 0:
        n = max(1, min(n, int((w >= float(min_p)).sum())))
    margin = 1.0
    if top_p < 1:
        c = np.cumsum(w[order[:n]])
        gaps = np.abs(c / c[-1] - float(top_p))
        n = min(n, 1 + int((c < float(top_p) * c[-1]).sum()))
        if not whole(w):
            margin = gaps[max(0, n - 2):n].min()
    return order[:n], w, margin


def whole(w) -> bool:
    """Weights of 0 and 1 alone: their sums are exact, and a border is where it is."""
    return bool(((w == 0) | (w == 1)).all())


def sample(x, u, **limits):
    """One row: token, log probability, and how near u is to another token or border (relative)."""
    order, w, margin = kept(x, **limits)
    if not len(order):
        return -1, -np.inf, 1.0
    places = np.sort(order)
    c = np.cumsum(w[places])
    i = min(int((c <= float(u) * c[-1]).sum()), len(places) - 1)
    if not whole(w):
        margin = min(margin, np.abs(c[:-1] / c[-1] - float(u)).min(initial=1.0))
    return int(places[i]), float(np.log(w[places[i]] / c[-1])), margin
