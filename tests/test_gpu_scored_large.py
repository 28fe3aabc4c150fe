"""Gradients of scored routing at the sizes that the persistent kernels, several token shares of dW and the wide fp32 tiles take,
against the fp64 oracle. Bounds as in test_gpu_route_scored: 2e-5 of the sum of the terms' magnitudes (dz in two bf16 parts for dx is
within 2^-17 of itself, 0.8e-5; an accumulator that is cut at each of its n / 16 steps, n up to 512 tokens or 256 experts, within
32 * 2^-23 = 0.4e-5), and 2^-8 of the value where it rounds to bf16."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M

from .test_gpu_route_scored import case, check, check_gradient, desc_of, run

pytestmark = pytest.mark.gpu

RULES = [dict(E=256, K=8, score="sigmoid", n_group=8, topk_group=4, group_top=2, scale=2.5),  # two 128-expert halves
         dict(E=100, K=3, renorm=False)]                                                       # dense dz, experts that end inside a tile


# (items of 128 tokens by 256 columns: 320, 306 and 171; more than the SMs, so that a CTA takes a second one and a third)
@pytest.mark.parametrize("rule", [0, 1])
@pytest.mark.parametrize("T,d", [(2500, 4096), (6500, 1472), (2305, 2240)])
def test_bf16(T, d, rule):
    one(T, d, rule, torch.bfloat16)


# (128-row tiles from 152 of them on: dx 160 and 152; dW of 256 experts in 10 planes 160)
@pytest.mark.parametrize("rule", [0, 1])
@pytest.mark.parametrize("T,d", [(2500, 512), (2400, 512)])
def test_fp32(T, d, rule):
    one(T, d, rule, torch.float32)


def one(T, d, rule, dtype):
    r = RULES[rule]
    kw = {k: v for k, v in r.items() if k not in ("E", "K")}
    x, w, ref = case(T + d, T, d, r["E"], r["K"], dtype, None, **kw)
    D = desc_of(d, r["E"], r["K"], dtype, **kw)
    idx, gate, logits, load = run(D, x, w)
    check(idx, gate, logits, load, ref)
    dg = torch.randn(T, r["K"], generator=torch.Generator().manual_seed(9))
    args = D, x.cuda(), w.cuda(), idx, gate, logits, dg.cuda()
    dx, dw = M.mcft_route_scored_grad(*args)
    M.mcft_device_error()
    check_gradient(dx, dw, x, w, ref, dg.double().numpy(), dtype, r.get("score", "softmax"), r.get("renorm", True), r.get("scale", 1.0))
    again = M.mcft_route_scored_grad(*args)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
