"""Pins of the fp64 oracle of the dense block, its 8-bit format and the norm: torch's e4m3 numbers, brute force, and central
differences."""
import numpy as np
import pytest
import torch

from oracle import dense


def test_grid_is_e4m3():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    assert np.array_equal(dense.GRID, codes.double().numpy())


def test_codes_by_brute_force():
    a = np.concatenate([np.random.default_rng(0).uniform(0, 448, 500), np.random.default_rng(1).uniform(0, 0.05, 500),
                        (dense.GRID[1:] + dense.GRID[:-1]) / 2, dense.GRID])
    far = np.abs(a[:, None] - dense.GRID)
    best = far.min(1)
    for v, c, b, f in zip(a, dense.round_to_grid(a), best, far):
        near = np.flatnonzero(f == b)
        assert c in near and (len(near) == 1 or c % 2 == 0), v


@pytest.mark.parametrize("big,s", [(448.0, 0), (np.nextafter(448.0, 449), 1), (224.0, -1), (1.75, -8), (1.0, -8), (3.5, -7),
                                   (0.0, -127), (2.0 ** -140, -127), (448 * 2.0 ** -127, -127), (3.4e38, 120)])
def test_scale_is_the_smallest_that_holds_the_block(big, s):
    assert dense.scale_exponent(big) == s
    assert big <= 448 * 2.0 ** s and (s == -127 or big > 448 * 2.0 ** (s - 1))


def test_blocks():
    x = np.random.default_rng(2).normal(size=(5, 71)) * np.exp(np.random.default_rng(3).normal(size=(5, 71)) * 4)
    x[1, 3], x[2, 40], x[3, :] = np.nan, -np.inf, 0.0
    v, codes, scales = dense.mx8(x)
    assert codes.shape == (5, 96) and scales.shape == (5, 3)
    assert np.isnan(v[1, :32]).all() and np.isfinite(v[1, 32:]).all() and scales[1, 0] == 255
    assert np.isnan(v[2, 32:64]).all() and scales[2, 1] == 255 and not v[3].any()
    ok = np.isfinite(v)
    assert (np.abs(v - np.where(ok, x, 0))[ok] <= dense.mx8_step(np.where(ok, x, 0))[ok] / 2).all()
    read = torch.from_numpy(codes.copy()).view(torch.float8_e4m3fn).double().numpy().reshape(5, 3, 32) * np.ldexp(1.0, scales.astype(int) - 127)[..., None]
    assert np.array_equal(read.reshape(5, 96)[:, :71][ok], v[ok])


def differences(f, x, h=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        out[i] = (f(a) - f(b)) / (2 * h)
    return out


def test_norm_gradient():
    r = np.random.default_rng(4)
    x, gamma, du, dres = r.normal(size=(3, 8)), r.normal(size=8), r.normal(size=(3, 8)), r.normal(size=(3, 8))
    loss = lambda x, gamma: (dense.norm(x, None, gamma, 1e-3)[1] * du).sum() + (x * dres).sum()  # noqa: E731
    dx, dgamma = dense.norm_grad(x, dense.norm(x, None, gamma, 1e-3)[2], gamma, du, dres)
    np.testing.assert_allclose(dx, differences(lambda v: loss(v, gamma), x), atol=1e-8)
    np.testing.assert_allclose(dgamma, differences(lambda v: loss(x, v), gamma), atol=1e-8)


def test_block_gradient():
    r = np.random.default_rng(5)
    x, dy = r.normal(size=(3, 4)), r.normal(size=(3, 4))
    w1, w3, w2 = r.normal(size=(5, 4)), r.normal(size=(5, 4)), r.normal(size=(4, 5))
    loss = lambda x, w1, w3, w2: (dense.ffn(x, w1, w3, w2)[0] * dy).sum()  # noqa: E731
    _, g, u, _ = dense.ffn(x, w1, w3, w2)
    dx, d1, d3, d2 = dense.ffn_grad(dy, w1, w3, w2, x, g, u)[:4]
    np.testing.assert_allclose(dx, differences(lambda v: loss(v, w1, w3, w2), x), atol=1e-8)
    np.testing.assert_allclose(d1, differences(lambda v: loss(x, v, w3, w2), w1), atol=1e-8)
    np.testing.assert_allclose(d3, differences(lambda v: loss(x, w1, v, w2), w3), atol=1e-8)
    np.testing.assert_allclose(d2, differences(lambda v: loss(x, w1, w3, v), w2), atol=1e-8)


def test_block_is_torchs():
    t = torch.Generator().manual_seed(6)
    x, dy = (torch.randn(7, 6, generator=t, dtype=torch.float64, requires_grad=q) for q in (True, False))
    w = [torch.randn(*s, generator=t, dtype=torch.float64, requires_grad=True) for s in ((9, 6), (9, 6), (6, 9))]
    y = (torch.nn.functional.silu(x @ w[0].T) * (x @ w[1].T)) @ w[2].T
    y.backward(dy)
    a = [v.detach().numpy() for v in (x, *w)]
    y2, g, u, _ = dense.ffn(*a)
    np.testing.assert_allclose(y2, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    for got, want in zip(dense.ffn_grad(dy.numpy(), *a[1:], a[0], g, u)[:4], (x, *w)):
        np.testing.assert_allclose(got, want.grad.numpy(), rtol=1e-11, atol=1e-11)
