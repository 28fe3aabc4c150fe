"""Scored routing and its gradient in fp64: z = W x, s = softmax(z) or sigmoid(z), choice by c = s + b within the
best groups, gates from s; gradient of sum(dgate * gate) with the choice held fixed."""
from __future__ import annotations

import numpy as np


def scores(z, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + np.exp(-z))
    e = np.exp(z - z.max(1, keepdims=True))
    return e / e.sum(1, keepdims=True)


def _best(v, k):
    """Indices of the k largest of a vector, largest first, equal ones by index."""
    return sorted(range(len(v)), key=lambda i: (-v[i], i))[:k]


def route(x, w, K, score="softmax", bias=None, n_group=1, topk_group=1, group_top=1, renorm=True, scale=1.0):
    """idx, gate, load, z, and `clear`: tokens whose decisions are apart by more than 1e-4 of the scores' size."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    s = scores(z, score)
    c = s if bias is None else s + np.asarray(bias, np.float64)
    T, E = z.shape
    gsz = E // n_group
    idx = np.full((T, K), -1, np.int32)
    gate = np.zeros((T, K))
    clear = np.ones(T, bool)
    for t in range(T):
        unit = 1e-4 * (np.sort(s[t])[::-1][min(K, E - 1)] + (0.01 if bias is not None else 0.0))
        groups = range(n_group)
        if n_group > 1:
            value = [np.sort(c[t, g * gsz:(g + 1) * gsz])[::-1][:group_top].sum() for g in range(n_group)]
            order = _best(value, n_group)
            groups = order[:topk_group]
            if topk_group < n_group:
                a, b = value[order[topk_group - 1]], value[order[topk_group]]
                clear[t] &= b == -np.inf or a - b > unit
        ok = [e for g in sorted(groups) for e in range(g * gsz, (g + 1) * gsz) if c[t, e] > -np.inf]
        order = [ok[i] for i in _best(c[t, ok], K + 1)] if ok else []
        clear[t] &= all(c[t, a] - c[t, b] > unit for a, b in zip(order, order[1:]))
        chosen = order[:K]
        idx[t, :len(chosen)] = chosen
        total = s[t, chosen].sum() if renorm else 1.0
        if total > 0:
            gate[t, :len(chosen)] = s[t, chosen] / total * scale
    load = np.bincount(idx[idx >= 0], minlength=E)
    return dict(idx=idx, gate=gate, load=load, z=z, s=s, clear=clear)


def gates(x, w, idx, score, renorm, scale):
    """The gates of a fixed choice."""
    s = scores(np.asarray(x, np.float64) @ np.asarray(w, np.float64).T, score)
    p = np.where(idx >= 0, np.take_along_axis(s, np.maximum(idx, 0).astype(np.int64), 1), 0.0)
    if renorm:
        p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
    return p * scale


def gradient(x, w, idx, dgate, score, renorm, scale):
    """dx, dw of sum(dgate * gates) through dgate -> ds -> dz, one Jacobian at a time."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    s = scores(x @ w.T, score)
    ds = np.zeros_like(s)
    for t in range(len(x)):
        on = [(int(e), k) for k, e in enumerate(idx[t]) if e >= 0]
        total = sum(s[t, e] for e, _ in on)
        mean = sum(s[t, e] * dgate[t, k] for e, k in on) / total if on else 0.0
        for e, k in on:
            ds[t, e] += scale * (dgate[t, k] - mean) / total if renorm else scale * dgate[t, k]
    if score == "sigmoid":
        dz = ds * s * (1 - s)
    elif renorm:
        dz = s * ds  # (sum_j s_j ds_j is 0 identically; fp64 would leave 1e-17 of it on every expert)
    else:
        dz = s * ds - s * (s * ds).sum(1, keepdims=True)
    return dz @ w, dz.T @ x
