"""Calls on a stream of their own, with the workspace left to the binding: memory that the current stream takes and fills while the
call's kernels wait is never the call's. Bits as on the current stream."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M

from .test_gpu_mx4_moe import Layer
from .test_gpu_route_scored import desc_of

pytestmark = pytest.mark.gpu


def on_a_busy_stream(call):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)  # about 10 ms
    out = call(s)
    filled = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in [1 << k for k in range(9, 25)] * 4]
    s.synchronize()
    M.mcft_device_error()
    del filled
    return out


@pytest.mark.parametrize("T", [3, 40, 300])
def test_layer(T):
    L = Layer(256, 8, 2, 512, 1)
    x, idx, gate = (t.cuda() for t in L.batch(T))
    want = L.run(x, idx, gate)
    got = on_a_busy_stream(lambda s: M.mcft_moe_forward_mx4(L.desc, x, idx, gate, L.blocks[:8], L.blocks[8:], stream=s))
    assert torch.equal(got, want)


@pytest.mark.parametrize("T", [3, 300])
def test_gradient(T):
    g = torch.Generator().manual_seed(T)
    x, w = torch.randn(T, 256, generator=g).bfloat16().cuda(), (torch.randn(64, 256, generator=g) * 0.1).bfloat16().cuda()
    D = desc_of(256, 64, 6, torch.bfloat16, renorm=False)
    logits = torch.empty(T, 64, device="cuda")
    idx, gate = M.mcft_route_scored(D, x, w, logits=logits)
    dg = torch.randn(T, 6, generator=g).cuda()
    want = M.mcft_route_scored_grad(D, x, w, idx, gate, logits, dg)
    torch.cuda.synchronize()
    got = on_a_busy_stream(lambda s: M.mcft_route_scored_grad(D, x, w, idx, gate, logits, dg, stream=s.cuda_stream))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
