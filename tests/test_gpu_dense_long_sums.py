"""The block's gradient over many tokens: sums of terms of one sign.

The tensor cores cut an accumulator's last bits towards zero at every step of 16 terms, up to 2^-23 of what it holds then. The
library therefore has an accumulator hold at most 2048 terms where the result stays fp32, 8192 where it is rounded to bf16, and adds
up the accumulators in fp32. Bounds for the terms below, positive multiples of 2^-15 under 4.7 whose runs of 2048 come to 5000 or so:
sums are exact up to 2^9, then a step of 38 or so costs up to 2^-14 (14 steps, to 2^10), 2^-13 (27, to 2^11), 2^-12 (54, to 2^12) and 2^-11
(24): 0.029 in all, 5.8e-6 of a run. The additions of n runs cost up to 2^-24 of half the total each in the mean: 1.0e-6 for the 32 runs
here. Together under 2^-17.
A run of 8192 terms costs up to 512 steps of 2^-23 of at most its sum: 2^-14."""
import numpy as np
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M
from tests.dense_model import Case, f64, near

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T", [4096, 65536, 65519])
def test_gradient_of_many_tokens(T):
    """dW2 = dy^T h with dy from 0.5 to 1.5 and h from 1.7 to 3.1 known to the bit: g = 2, u of four values, h their product rounded
    to bf16 (no product lies near the middle between two bf16 numbers). Large enough that the contraction is not split over the SMs."""
    d = w = 2048
    D = M.LayerDesc(d, 0, 0, w, 0, 0, M.MCFT_BF16)
    gen = torch.Generator(device="cuda").manual_seed(T)
    u = 1 + 0.25 * torch.randint(0, 4, (T, w), generator=gen, device="cuda")
    gu = torch.cat((torch.full((T, w), 2.0, device="cuda"), u), 1)
    ckpt = M.mcft_mx8_quantize(gu)
    assert torch.equal(M.mcft_mx8_dequantize(ckpt, T, 2 * w, F32), gu)
    del gu
    values = 2 / (1 + np.exp(-2.0)) * np.array([1, 1.25, 1.5, 1.75])
    place = values / 2.0 ** (np.floor(np.log2(values)) - 7)
    assert (np.abs(place - np.floor(place) - 0.5) > 2.0 ** -7).all()  # (the kernel's h is within 2^-20 of itself before it is rounded)
    h = (2 / (1 + np.exp(-2.0)) * u.double()).bfloat16()
    dy = (0.5 + torch.rand(T, d, generator=gen, device="cuda")).bfloat16()
    block = torch.randn(3 * w * d, generator=gen, device="cuda").bfloat16()
    x = torch.randn(T, d, generator=gen, device="cuda").bfloat16()
    _, full = M.mcft_ffn_grad(D, dy, block, x=x, ckpt=ckpt, grad_dtype=F32)
    _, half = M.mcft_ffn_grad(D, dy, block, x=x, ckpt=ckpt)
    M.mcft_ffn_grad(D, dy, block, x=x, ckpt=ckpt, dblock=full, accumulate=True)
    M.mcft_device_error()
    rows = torch.arange(0, d, 61, device="cuda")
    want = dy[:, rows].double().T @ h.double()
    got = full[2 * w * d:].view(d, w)[rows].double()
    off = ((got - 2 * want) / (2 * want)).abs().max().item()
    assert off <= 2.0 ** -17 + 2.0 ** -24, off
    # rounding keeps order: between the roundings of the smallest and the largest sum that the runs may leave
    low, high = (want * (1 - 2.0 ** -14 - 2.0 ** -20)).bfloat16(), (want * (1 + 2.0 ** -20)).bfloat16()
    got = half[2 * w * d:].view(d, w)[rows]
    assert bool(((low <= got) & (got <= high)).all()), (got < low).float().mean().item()
    _, twice = M.mcft_ffn_grad(D, dy, block, x=x, ckpt=ckpt, dblock=half.clone(), accumulate=True)
    low, high = ((got.double() + want * (1 + e)).bfloat16() for e in (-2.0 ** -14 - 2.0 ** -20, 2.0 ** -20))
    got = twice[2 * w * d:].view(d, w)[rows]
    assert bool(((low <= got) & (got <= high)).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d,w", [(700, 192, 4096), (700, 320, 4160), (150, 64, 12352), (8200, 64, 64), (10000, 320, 4224), (20000, 2048, 8256)])
def test_forward_and_gradient_around_a_run(T, d, w, dtype):
    """Contractions of one run, a run and a bit, several, and split ones, against the model's bounds (terms of either sign), or
    where fp64 would take long some rows of y and dx against fp64 sums of the operands that the kernels round."""
    if T * d * w > 1e10 and dtype == F32:
        return  # (fp32 layers have shorter runs at any size)
    if T * d * w > 2e10:
        D = M.LayerDesc(d, 0, 0, w, 0, 0, M.MCFT_BF16)
        gen = torch.Generator(device="cuda").manual_seed(1)
        x, dy = (torch.randn(T, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
        block = (torch.randn(3 * w * d, generator=gen, device="cuda") / d ** 0.5).bfloat16()
        y = M.mcft_ffn_forward(D, x, block)
        dx, db = M.mcft_ffn_grad(D, dy, block, x=x, grad_dtype=F32)
        w1, w3, w2 = block[:w * d].view(w, d), block[w * d: 2 * w * d].view(w, d), block[2 * w * d:].view(d, w)
        t = torch.arange(7, T, 397, device="cuda")
        g, u = x[t].double() @ w1.double().T, x[t].double() @ w3.double().T
        s, dh, r = torch.sigmoid(g), dy[t].double() @ w2.double(), lambda v: v.bfloat16().double()  # noqa: E731
        want = r(g * s * u) @ w2.double().T, r(dh * u * s * (1 + g * (1 - s))) @ w1.double() + r(dh * g * s) @ w3.double()
        # (the operands are the kernel's but where fp32 moved one over a middle; outputs within half a bf16 step of themselves)
        for a, b in zip((y, dx), want):
            assert ((a[t].double() - b).norm() / b.norm()).item() < 2.0 ** -8
        again = (M.mcft_ffn_forward(D, x, block), *M.mcft_ffn_grad(D, dy, block, x=x, grad_dtype=F32))
        assert all(torch.equal(a, b) for a, b in zip(again, (y, dx, db)))
        return
    c = Case(T, d, w, dtype, 3)
    D = M.LayerDesc(d, 0, 0, w, 0, 0, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32)
    near(M.mcft_ffn_forward(D, c.x, c.block), *c.forward(), "y")
    dx, db = M.mcft_ffn_grad(D, c.dy, c.block, x=c.x)
    M.mcft_device_error()
    (wx, rx), (wb, rb) = c.gradient(f64(c.x), *c.projections(f64(c.x)))
    near(dx, wx, rx, "dx")
    near(db, wb, rb, "dblock")
