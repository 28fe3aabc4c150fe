"""The mx4 layer's weighted sum: fp32 terms, one rounding of y, so that experts whose outputs nearly cancel leave their
difference and not what a rounding of each of them leaves.

Two experts have the same gate and up weights and down weights that differ in the sign of one column j alone, and every token
takes them with gates g and -g: y = 2 g W2[:, j] h[j]. Tolerance: h[j] may round either way where it is close to a tie (the
oracle's slack); each expert's fp32 sums are within 2^-18 of its row's largest output, as in test_gpu_mx4_moe; and y rounds to
bf16, 2^-8 of itself."""
import numpy as np
import pytest
import torch

import oracle.mx4 as O
from paper_2609_34077_gb300 import mcft as M
from .test_gpu_mx4_moe import Layer

pytestmark = pytest.mark.gpu


def hidden(x, w1, w3):
    """h before its rounding, and how far fp32 sums may move it (as oracle.mx4.expert_forward)."""
    xq, q1, q3 = O.quantize(x), O.quantize(w1), O.quantize(w3)
    g, u = xq @ q1.T, xq @ q3.T
    s = g / (1.0 + np.exp(-g))
    dg, du = 2.0 ** -22 * (np.abs(xq) @ np.abs(q1).T), 2.0 ** -22 * (np.abs(xq) @ np.abs(q3).T)
    return s * u, 1.1 * dg * np.abs(u) + np.abs(s) * du + 2.0 ** -21 * np.abs(s * u)


# 20 tokens: one tile for all; 130 and 300: permuted; 24 experts of 2048 outputs: up to 26 tiles of eight column ranges
@pytest.mark.parametrize("T", [1, 20, 130, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_that_cancel(T, dtype):
    d, w, E, j, g = 2048, 256, 24, 37, 0.75
    L = Layer(d, E, 2, w, 0, dtype, seed=5)
    other = L.plain[0].clone()
    other[2 * w * d:].view(d, w)[:, j] *= -1
    L.blocks[1] = M.mcft_mx4_pack_expert(L.desc, other.cuda())
    x, idx, gate = L.batch(T)
    idx[:, 0], idx[:, 1] = 0, 1
    gate[:, 0], gate[:, 1] = g, -g
    y = L.run(x, idx, gate).cpu().double().numpy()
    w1, w3, w2 = L.triples[0]
    h, dh = hidden(x.double().numpy(), w1, w3)
    hq, room, q2 = O.quantize(h), O.slack(h, dh), O.quantize(w2)
    ref = 2 * g * hq[:, j:j + 1] * q2[None, :, j]
    tol = 2 * g * room[:, j:j + 1] * np.abs(q2[None, :, j]) + 2 * g * 2.0 ** -18 * np.abs(hq @ q2.T).max(1, keepdims=True)
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(ref)
    err = np.abs(y - ref)
    assert (err <= tol + 1e-30).all(), f"worst {np.max(err / (tol + 1e-30)):.3g} of the bound"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_token_gives_the_same_bits_in_larger_batches(dtype):
    """Permuted batches of any size, by single tiles and by pairs, add the same sums."""
    L = Layer(2048, 2, 1, 2560, 1, dtype)
    x, idx, gate = L.batch(1500, drop=0.1)
    y = L.run(x, idx, gate)
    for at in (0, 300, 1200):
        part = slice(at, at + 300)
        assert torch.equal(y[part], L.run(x[part], idx[part], gate[part]))
