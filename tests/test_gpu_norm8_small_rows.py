"""RMSNorm with mx8 outputs where mean v^2 + eps is a subnormal fp32 number, with its gradient: 1 / sqrt of it is finite (up to 2^74.5).

Tolerances. Below 2^-126 a thread's squares are rounded to multiples of 2^-149, each by at most 2^-150, and so are their mean's
quotient and the eps of the caller; sums of such multiples are exact. So mean + eps is off by at most 2^-149 beside the 2^-23 that r
is off by elsewhere: r and u by the share 2^-149 / (mean + eps) of themselves, for shares up to a half (1 / sqrt(1 - e) <= 1 + e)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_34077_gb300 import mcft as M

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SIZES = [3e-19, 6e-20, 5e-20, 2e-20, 1e-20, 1e-21, 1e-22]


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-40, 2e-39])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 4160, 16448])
def test_rows_of_subnormal_squares(d, dtype, eps):
    g = torch.Generator().manual_seed(d)
    x = torch.randn(len(SIZES) + (eps > 0), d, generator=g)
    x[:len(SIZES)] *= torch.tensor(SIZES)[:, None]
    x[len(SIZES):] = 0.0  # (u = 0: r is that of eps alone)
    gamma = (1 + 0.2 * torch.randn(d, generator=g)).to(dtype)
    du = torch.randn(x.shape, generator=g).to(dtype)
    D = M.LayerDesc(d, 0, 0, 0, 0, 0, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32)
    out, u, u8, rstd = M.mcft_residual_rmsnorm_mx8(D, x.cuda(), None, gamma.cuda(), eps)
    dx, dgamma = M.mcft_rmsnorm_grad(D, gamma.cuda(), rstd, du.cuda(), x=out)
    back = M.mcft_mx8_dequantize(u8, len(x), d, F32)
    M.mcft_device_error()
    v = f64(x)
    mean = (v * v).mean(1) + float(np.float32(eps))
    r = 1 / np.sqrt(mean)
    share = 2.0 ** -149 / mean
    assert (share < 0.5).all()
    off = np.abs(f64(rstd) - r)
    assert (off <= r * (2.0 ** -23 + share)).all(), off / r
    want = v * r[:, None] * f64(gamma)
    room = np.abs(want) * (2.0 ** -22 + share[:, None])
    assert (np.abs(f64(u) - want) <= room + np.abs(want) * (2.0 ** -8 if dtype == BF16 else 0)).all()
    assert (np.abs(f64(back) - want) <= room + 0.5 * oracle.dense.mx8_step(np.abs(want) + room)).all()
    # the gradient takes r as it is: bounds as for other rows
    n = v * f64(rstd)[:, None]
    wx, wg = oracle.dense.norm_grad(v, f64(rstd), f64(gamma), f64(du), None)
    gd = np.abs(f64(gamma) * f64(du))
    room = np.abs(wx) * 2.0 ** -23 + f64(rstd)[:, None] * (gd + np.abs(n) * (gd * np.abs(n)).mean(1, keepdims=True)) * 2.0 ** -18
    assert (np.abs(f64(dx) - wx) <= room).all()
    assert (np.abs(f64(dgamma) - wg) <= (np.abs(f64(du)) * np.abs(n)).sum(0) * 2.0 ** -18).all()
