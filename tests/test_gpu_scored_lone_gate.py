"""A gate that is renormalised alone is the constant `scale`: its gradient is 0, not what rounding leaves of it."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M

from .test_gpu_route_scored import desc_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,dtype", [(37, torch.float32), (700, torch.bfloat16)])
@pytest.mark.parametrize("K,bias", [(1, False), (3, True)])
def test_no_gradient(score, T, dtype, K, bias):
    d, E = 320, 24
    g = torch.Generator().manual_seed(T + K)
    x, w = torch.randn(T, d, generator=g).to(dtype).cuda(), (torch.randn(E, d, generator=g) * 0.1).to(dtype).cuda()
    b = None
    if bias:  # all experts but one are out: K - 1 of the choices are empty
        b = torch.full((E,), float("-inf"), device="cuda")
        b[17] = 0.0
    desc = desc_of(d, E, K, dtype, score, scale=2.5)
    logits = torch.empty(T, E, device="cuda")
    idx, gate = M.mcft_route_scored(desc, x, w, b, logits=logits)
    assert (gate[:, 0] == 2.5).all() and (gate[:, 1:] == 0).all()
    dgate = torch.randn(T, K, generator=g).cuda()
    dx, dw = M.mcft_route_scored_grad(desc, x, w, idx, gate, logits, dgate)
    M.mcft_device_error()
    assert (dx == 0).all() and (dw == 0).all()
