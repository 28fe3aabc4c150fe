"""The dense gated feed-forward block, its 8-bit checkpoints and the RMSNorm ahead of it, forward and backward, in fp64.

mx8, from the definition: blocks of 32 along a row under 2^s, s the smallest in [-127, 127] with max|x| <= 448 * 2^s; values
rounded to the nearest e4m3 number (sign, four exponent bits of bias 7, three mantissa bits, subnormals of 2^-9, 448 the largest),
ties to the even code, or to 1.875 * 2^127 where that would be 2^128 (fp32 and bf16 end below); a block with a NaN or an infinity
is NaN."""
from __future__ import annotations

import numpy as np

# the non-negative e4m3 numbers in order of their codes 0 .. 126
GRID = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def round_to_grid(a):
    """Code of the nearest e4m3 number of a in [0, 448], ties to the even code."""
    hi = np.minimum(np.searchsorted(GRID, a, side="left"), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    return np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))


def scale_exponent(big):
    """Smallest s in [-127, 127] with big <= 448 * 2^s."""
    m, e = np.frexp(np.asarray(big, np.float64) / 448.0)  # big / 448 = m 2^e, m in [0.5, 1)
    return np.where(big > 0, np.clip(np.where(m == 0.5, e - 1, e), -127, 127), -127)


def mx8(x):
    """(values, codes, scale bytes) of x [R, C]; codes and bytes as they stand in an mx8 matrix."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    v = np.zeros((R, -(-C // 32) * 32))
    v[:, :C] = x
    v = v.reshape(R, -1, 32)
    ok = np.isfinite(v).all(2, keepdims=True)
    v = np.where(ok, v, 0.0)
    s = scale_exponent(np.abs(v).max(2, keepdims=True))
    unit = np.ldexp(1.0, s)
    code = np.where(s == 120, np.minimum(round_to_grid(np.abs(v) / unit), 0x77), round_to_grid(np.abs(v) / unit))
    values = np.where(ok, np.copysign(GRID[code] * unit, v), np.nan).reshape(R, -1)[:, :C]
    codes = np.where(np.signbit(v), code + 128, code).reshape(R, -1)
    return values, codes.astype(np.uint8), np.where(ok, s + 127, 255)[..., 0].astype(np.uint8)


def mx8_step(x):
    """The largest distance between neighbouring numbers of the format at each value of x, under its block's scale."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    v = np.zeros((R, -(-C // 32) * 32))
    v[:, :C] = np.abs(x)
    v = v.reshape(R, -1, 32)
    unit = np.ldexp(1.0, scale_exponent(v.max(2, keepdims=True)))
    e = np.maximum(np.floor(np.log2(np.maximum(v / unit, 2.0 ** -9))), -6)
    return (np.ldexp(unit, (e - 3).astype(int))).reshape(R, -1)[:, :C]


def norm(x, y, gamma, eps):
    """(v = x + y, u, rstd)."""
    v = x if y is None else x + y
    r = 1.0 / np.sqrt((v * v).mean(1) + eps)
    return v, gamma * v * r[:, None], r


def norm_grad(v, rstd, gamma, du, dres):
    """(dv, dgamma) of a loss that reaches v through the norm (rstd as a function of v) and past it by dres."""
    n = v * rstd[:, None]
    g = gamma * du
    dv = rstd[:, None] * (g - n * (g * n).mean(1, keepdims=True))
    return dv + (0.0 if dres is None else dres), (du * n).sum(0)


def sigmoid(g):
    return np.where(g >= 0, 1.0 / (1.0 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1.0 + np.exp(-np.abs(g))))


def ffn(x, w1, w3, w2):
    """(y, g, u, h)."""
    g, u = x @ w1.T, x @ w3.T
    h = g * sigmoid(g) * u
    return h @ w2.T, g, u, h


def ffn_grad(dy, w1, w3, w2, x, g, u):
    """(dx, dW1, dW3, dW2, and dg, du, h) from dy and the forward's x, g and u."""
    s = sigmoid(g)
    h, dh = g * s * u, dy @ w2
    du, dg = dh * g * s, dh * u * s * (1.0 + g * (1.0 - s))
    return dg @ w1 + du @ w3, dg.T @ x, du.T @ x, dy.T @ h, dg, du, h
