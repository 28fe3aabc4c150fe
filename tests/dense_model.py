"""The dense block in fp64 with elementwise bounds of what the library's arithmetic may be off by.

f: what an fp32 sum may be off by, relative to the sum of its terms' magnitudes: at most n 2^-24 for n terms added in turn, of
which rounding errors of either sign leave far less; the tensor cores cut an accumulator's last bits towards zero, a bias of 1.2e-6 =
2^-19.7 at 4096 terms. Taken: 2^-18 (bf16), 2^-20 (fp32 multiply-adds, whose errors have either sign).
r: half a step of an operand or output that is rounded to bf16, 2^-8 of its value (fp32: 2^-23 for the last operation).
SwiGLU's own arithmetic: within 2^-20 of its value. |silu'| <= 1.1, |silu''| <= 0.5."""
import numpy as np
import torch

import oracle


def f64(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, T, d, w, dtype, seed=0):
        g = torch.Generator().manual_seed(seed + 7 * T + d + w)
        self.T, self.d, self.w, self.dtype = T, d, w, dtype
        self.x = torch.randn(T, d, generator=g).to(dtype).cuda()
        self.dy = (0.1 * torch.randn(T, d, generator=g)).to(dtype).cuda()
        self.block = (torch.randn(3 * w * d, generator=g) * (1.3 / d ** 0.5)).to(dtype).cuda()
        n = w * d
        b = f64(self.block)
        self.w1, self.w3, self.w2 = b[:n].reshape(w, d), b[n: 2 * n].reshape(w, d), b[2 * n:].reshape(d, w)
        self.f = 2.0 ** -18 if dtype == torch.bfloat16 else 2.0 ** -20
        self.r = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23

    def projections(self, x):
        """g, u of x and their bounds."""
        ax = np.abs(x)
        return x @ self.w1.T, x @ self.w3.T, self.f * (ax @ np.abs(self.w1).T), self.f * (ax @ np.abs(self.w3).T)

    def hidden(self, g, u, eg, eu):
        """h, its bound with the operand's rounding."""
        a = g * oracle.dense.sigmoid(g)
        h = a * u
        return h, 1.1 * eg * (np.abs(u) + eu) + np.abs(a) * eu + (2.0 ** -20 + self.r) * np.abs(h)

    def forward(self):
        """y and its bound."""
        g, u, eg, eu = self.projections(f64(self.x))
        h, eh = self.hidden(g, u, eg, eu)
        y, a2 = h @ self.w2.T, np.abs(self.w2).T
        return y, eh @ a2 + self.f * (np.abs(h) @ a2) + self.r * np.abs(y)

    def gradient(self, x, g, u, eg=0.0, eu=0.0, out_r=None):
        """(dx, dblock) and their bounds, from values of x, g and u (g and u off by up to eg and eu)."""
        r = self.r if out_r is None else out_r
        dy = f64(self.dy)
        dx, d1, d3, d2, dg, du, h = oracle.dense.ffn_grad(dy, self.w1, self.w3, self.w2, x, g, u)
        dh, edh = np.abs(dy @ self.w2), self.f * (np.abs(dy) @ np.abs(self.w2))
        au, a = np.abs(u) + eu, np.abs(g * oracle.dense.sigmoid(g))
        _, eh = self.hidden(g, u, eg, eu)
        edu = edh * (a + 1.1 * eg) + dh * 1.1 * eg + (2.0 ** -20 + self.r) * np.abs(du)
        edg = 1.1 * edh * au + 1.1 * dh * eu + 0.5 * dh * au * eg + 2.0 ** -20 * dh * au + self.r * np.abs(dg)
        e = np.abs
        rx = edg @ e(self.w1) + edu @ e(self.w3) + self.f * (e(dg) @ e(self.w1) + e(du) @ e(self.w3)) + self.r * e(dx)
        r1 = edg.T @ e(x) + self.f * (e(dg).T @ e(x)) + r * e(d1)
        r3 = edu.T @ e(x) + self.f * (e(du).T @ e(x)) + r * e(d3)
        r2 = e(dy).T @ eh + self.f * (e(dy).T @ e(h)) + r * e(d2)
        flat = lambda *m: np.concatenate([v.ravel() for v in m])  # noqa: E731
        return (dx, rx), (flat(d1, d3, d2), flat(r1, r3, r2))


def near(got, want, room, what=""):
    got = f64(got)
    assert got.shape == want.shape, what
    off = np.abs(got - want) - room
    assert np.isfinite(got).all() and (off <= 0).all(), f"{what}: {off.max():.3g} over the bound, {(off > 0).mean():.3g} of the values"
