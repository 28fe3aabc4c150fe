"""Microscaled 4-bit floating point in fp64: rounding to the format, the product of two rounded matrices, and
the routed layer on rounded weights and activations. Written from the definition: blocks of 32 along a row,
scale 2^(floor(log2 max|x|) - 2) clamped to [2^-127, 2^127], values rounded to the nearest of
0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even code), larger ones to 6; a block with a NaN or an infinity is NaN."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_to_grid(a):
    """Nearest grid value of a >= 0, ties to the even code."""
    a = np.asarray(a, np.float64)
    hi = np.minimum(np.searchsorted(GRID, a, side="left"), 7)  # GRID[hi] >= a, but past the end
    lo = np.maximum(hi - 1, 0)
    up = GRID[hi] - a
    down = a - GRID[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return GRID[np.where(a >= 6, 7, code)]


def _round(v, big, ok):
    """Blocks v [R, n] rounded under the scales that block maxima `big` give; zeros where not ok."""
    e = np.frexp(np.where((big > 0) & ok, big, 1.0))[1] - 1  # floor(log2)
    e = np.where(big > 0, e, -125)
    unit = np.ldexp(1.0, np.clip(e - 2, -127, 127))[:, None]
    return np.copysign(round_to_grid(np.abs(np.where(ok[:, None], v, 0.0)) / unit) * unit, v)


def quantize(x):
    """x [R, C] rounded to mx4, as fp64 values."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    for c in range(0, x.shape[1], 32):
        v = x[:, c:c + 32]
        ok = np.isfinite(v).all(1)
        out[:, c:c + 32] = np.where(ok[:, None], _round(v, np.abs(v).max(1), ok), np.nan)
    return out


def slack(x, delta):
    """How far the rounding of x can move when each of its elements moves by up to delta: over both ends of the
    element's range under the scales of both ends of its block's largest magnitude (rounding is monotone)."""
    base = quantize(x)
    out = np.zeros_like(base)
    for c in range(0, x.shape[1], 32):
        v, d = x[:, c:c + 32], delta[:, c:c + 32]
        big = np.abs(v).max(1)
        ok = np.ones(len(v), bool)
        for edge in (np.maximum(np.max(np.abs(v) - d, axis=1), 0.0), np.max(np.abs(v) + d, axis=1)):
            for w in (v - d, v + d):
                out[:, c:c + 32] = np.maximum(out[:, c:c + 32], np.abs(_round(w, edge, ok) - base[:, c:c + 32]))
        assert np.isfinite(big).all()
    return out


def expert_forward(x, w1, w3, w2):
    """F(x) = W2 Q(silu(W1 Q(x)) * (W3 Q(x))) with the three matrices rounded too, and how far F can move where
    the gate and up products are fp32 sums: each within 2^-22 of the sum of its terms' magnitudes (n terms of
    one sign at n 2^-24 would be more; sums of mixed signs wander by its root), silu within 2^-21 of itself."""
    xq, q1, q3, q2 = quantize(x), quantize(w1), quantize(w3), quantize(w2)
    g, u = xq @ q1.T, xq @ q3.T
    dg, du = 2.0 ** -22 * (np.abs(xq) @ np.abs(q1).T), 2.0 ** -22 * (np.abs(xq) @ np.abs(q3).T)
    with np.errstate(over="ignore"):
        s = g / (1.0 + np.exp(-g))
    h = s * u
    dh = 1.1 * dg * np.abs(u) + np.abs(s) * du + 2.0 ** -21 * np.abs(h)  # |silu'| <= 1.1
    return quantize(h) @ q2.T, slack(h, dh) @ np.abs(q2).T


def moe_layer(x, idx, gate, experts, shared=()):
    """Weighted sum of the selected experts (an idx of -1 is none) and the shared ones; and its slack."""
    x = np.asarray(x, np.float64)
    y, room = np.zeros_like(x), np.zeros_like(x)
    for e, blk in enumerate(experts):
        t, k = np.nonzero(np.asarray(idx) == e)
        if len(t):
            g = np.asarray(gate, np.float64)[t, k][:, None]
            f, r = expert_forward(x[t], *blk)
            np.add.at(y, t, g * f)
            np.add.at(room, t, np.abs(g) * r)
    for blk in shared:
        f, r = expert_forward(x, *blk)
        y, room = y + f, room + r
    return y, room
