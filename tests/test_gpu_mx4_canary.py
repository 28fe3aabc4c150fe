"""Out-of-bounds writes of the mx4 operators and of scored routing: every output and workspace sits between guard
regions that must be untouched after the call, each buffer of exactly the size the library asks for."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M
from tests.test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def guarded(guards, dtype, *shape):
    n = 1
    for s in shape:
        n *= s
    g = Guarded(n * torch.empty(0, dtype=dtype).element_size())
    guards.append(g)
    return g.view(dtype, shape)


def check(guards, what):
    M.mcft_device_error()
    for i, g in enumerate(guards):
        g.check(f"{what}, buffer {i}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,C", [(1, 1), (9, 33), (128, 256), (200, 1000), (257, 4097)])
def test_quantise_and_back(R, C, dtype):
    guards = []
    q = guarded(guards, torch.uint8, M.mcft_mx4_size(R, C))
    y = guarded(guards, dtype, R, C)
    M.mcft_mx4_quantize(torch.randn(R, C, device="cuda").to(dtype), q)
    M.mcft_mx4_dequantize(q, R, C, y=y)
    check(guards, f"{R} x {C}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M_,N,K", [(1, 65, 96), (3, 4096, 2048), (129, 200, 64), (1300, 2500, 160), (2048, 2432, 64)])
def test_product(M_, N, K, dtype):
    guards = []
    a, b = (guarded(guards, torch.uint8, M.mcft_mx4_size(r, K)) for r in (M_, N))
    M.mcft_mx4_quantize(torch.randn(M_, K, device="cuda"), a)
    M.mcft_mx4_quantize(torch.randn(N, K, device="cuda"), b)
    M.mcft_mx4_matmul(a, b, M_, N, K, y=guarded(guards, dtype, M_, N))
    check(guards, f"{M_} x {N} x {K}")


@pytest.mark.parametrize("T", [1, 13, 16, 17, 128, 129, 500])
@pytest.mark.parametrize("d,E,K,w,S", [(192, 10, 3, 320, 2), (128, 64, 6, 64, 0), (2048, 8, 2, 512, 1)])
def test_layer(T, d, E, K, w, S):
    guards = []
    desc = M.LayerDesc(d, E, K, w, S, M.MCFT_GATE_RENORM, M.MCFT_BF16)
    blocks = [M.mcft_mx4_pack_expert(desc, (torch.randn(3 * w * d, device="cuda") * 0.05).bfloat16(),
                                     guarded(guards, torch.uint8, M.mcft_mx4_expert_size(desc))) for _ in range(E + S)]
    idx = torch.rand(T, E, device="cuda").topk(K).indices.int()
    idx[::5, 0] = -1
    M.mcft_moe_forward_mx4(desc, torch.randn(T, d, device="cuda").bfloat16(), idx, torch.rand(T, K, device="cuda"), blocks[:E],
                           blocks[E:], y=guarded(guards, BF16, T, d),
                           workspace=guarded(guards, torch.uint8, M.mcft_mx4_workspace_size(desc, T)))
    check(guards, f"T = {T}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 5, 64, 65, 129, 300])
@pytest.mark.parametrize("d,E,K", [(64, 1, 1), (192, 33, 5), (2048, 256, 8)])
def test_scored_routing(T, d, E, K, dtype):
    guards = []
    desc = M.ScoredDesc(d, E, K, 1, 1, 1, M.MCFT_SCORE_SIGMOID, M.MCFT_GATE_RENORM, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32, 1.0)
    x, w = torch.randn(T, d, device="cuda").to(dtype), torch.randn(E, d, device="cuda").to(dtype)
    idx, gate = guarded(guards, torch.int32, T, K), guarded(guards, F32, T, K)
    logits, load = guarded(guards, F32, T, E), guarded(guards, torch.int32, E)
    M.mcft_route_scored(desc, x, w, idx=idx, gate=gate, logits=logits, load=load)
    M.mcft_route_scored_grad(desc, x, w, idx, gate, logits, torch.randn(T, K, device="cuda"), dx=guarded(guards, dtype, T, d),
                             dw=guarded(guards, F32, E, d),
                             workspace=guarded(guards, torch.uint8, M.mcft_route_scored_grad_workspace_size(desc, T)))
    check(guards, f"T = {T}")


@pytest.mark.parametrize("shape", [(256, 8, 2, 512, 0), (2048, 64, 6, 1408, 2), (64, 1, 1, 64, 8), (128, 256, 16, 64, 0)])
@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
def test_a_workspace_serves_any_fewer_tokens(shape, dtype):
    """(the sizes depend on the device's SMs)"""
    d, E, K, w, S = shape
    desc = M.LayerDesc(d, E, K, w, S, 0, dtype)
    scored = M.ScoredDesc(d, E, K, 1, 1, 1, 0, 0, dtype, 1.0)
    tokens = list(range(0, 1400)) + list(range(1400, 9000, 97))
    for sizes in ([M.mcft_mx4_workspace_size(desc, T) for T in tokens], [M.mcft_route_scored_grad_workspace_size(scored, T) for T in tokens]):
        assert sizes == sorted(sizes)
