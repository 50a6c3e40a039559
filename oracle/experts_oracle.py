"""CPU oracle for 8-bit linear layers and layers made of experts.

TEST INFRASTRUCTURE ONLY: imported by the tests, never by the library.  Plain
numpy in float64.

    row       s = max|x| / 127, q = x / s before its rounding to a whole number
    product   s_a[m] s_w[n] sum_k qa[m, k] qw[k, n], the sum in whole numbers
    routing   softmax or sigmoid; choice by score + bias within the best groups
    experts   slot i of expert e is row rows[i] by weight e
    sum       add[t] + sum_j w[t, j] y[places[t, j]]
"""
from __future__ import annotations

import numpy as np

__all__ = ["gated_rows", "row_codes", "w8a8", "route", "expert_order", "expert_products", "combine"]


def gated_rows(x):
    """silu of the first half of each row times the second."""
    g, u = np.split(np.asarray(x, np.float64), 2, axis=-1)
    return g / (1.0 + np.exp(-g)) * u


def row_codes(x):
    """(codes before rounding, scale) of each row; NaN where a value is not finite,
    zeros for rows under 2^-100."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(x).all(-1)
        none = top < 2.0 ** -100
        unit = np.where(bad | none, 1.0, top / 127)
        v = np.where((bad | none)[:, None], 0.0, x / unit[:, None])
    return v, np.where(bad, np.nan, np.where(none, 0.0, unit))


def w8a8(q, s, w, ws):
    """[M, N] in float64 of int8 codes [M, K] and [K, N]; sums below 2^53 are exact."""
    return (q.astype(np.float64) @ w.astype(np.float64)) * np.asarray(s, np.float64)[:, None] * np.asarray(ws, np.float64)


def route(logits, k, bias=None, scoring="softmax", groups=1, top_groups=None, group_score="top2", renormalize=False,
          scale=1.0):
    """(weights [T, k], experts [T, k]), one token at a time."""
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    top_groups = groups if top_groups is None else top_groups
    weights, experts = np.zeros((T, k)), np.zeros((T, k), np.int64)
    for t in range(T):
        row = np.where(np.isnan(x[t]), -np.inf, x[t])
        masked = row == -np.inf
        with np.errstate(over="ignore"):
            if scoring == "sigmoid":
                score = 1.0 / (1.0 + np.exp(-row))
            elif masked.all():
                score = np.zeros(E)
            elif row.max() == np.inf:
                score = (row == np.inf).astype(np.float64)
            else:
                score = np.exp(row - row.max())
        if scoring == "softmax" and score.sum() > 0:
            score = score / score.sum()
        choice = score + (0.0 if bias is None else np.asarray(bias, np.float64))
        masked |= np.isnan(choice) | (choice == -np.inf)
        choice = np.where(masked, -np.inf, choice)
        part = np.arange(E) // (E // groups)
        value = []
        for g in range(groups):
            seen = sorted(choice[(part == g) & ~masked], reverse=True)
            value.append(-np.inf if not seen else sum(seen[:2]) if group_score == "top2" else seen[0])
        best = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
        order = sorted((e for e in range(E) if part[e] in best), key=lambda e: (-choice[e], e))[:k]
        w = np.array([0.0 if masked[e] else score[e] for e in order])
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else np.zeros(k)
        weights[t], experts[t] = w * scale, order
    return weights, experts


def expert_order(experts, E):
    """(offsets [E + 1], tokens [T k], places [T, k]): choices by expert, then token."""
    T, k = experts.shape
    slots = [(e, t, j) for t in range(T) for j, e in enumerate(experts[t])]
    slots.sort()
    tokens = np.array([t for _, t, _ in slots], np.int64)
    places = np.zeros((T, k), np.int64)
    for i, (_, t, j) in enumerate(slots):
        places[t, j] = i
    counts = np.bincount(np.asarray(experts).ravel(), minlength=E)
    return np.concatenate([[0], np.cumsum(counts)]), tokens, places


def expert_products(q, s, w, ws, offsets, rows):
    """[slots, N]; NaN in rows that no expert has."""
    out = np.full((len(rows), w.shape[2]), np.nan)
    for e in range(w.shape[0]):
        for i in range(offsets[e], offsets[e + 1]):
            r = rows[i]
            out[i] = w8a8(q[r:r + 1], s[r:r + 1], w[e], ws[e])[0] if 0 <= r < len(q) else 0.0
    return out


def combine(y, weights, places, add=None):
    out = np.zeros((places.shape[0], y.shape[1])) if add is None else np.array(add, np.float64)
    for t in range(places.shape[0]):
        for w, p in zip(weights[t], places[t]):
            if w != 0 and 0 <= p < len(y):
                out[t] += w * y[p]
    return out
