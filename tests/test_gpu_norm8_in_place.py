"""The norm and its gradient over their own inputs, where the header allows it: the bits of separate buffers, at row widths of one and
several steps a thread, with rows that end inside a team's steps."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(1, 64), (33, 192), (1000, 320), (700, 2112), (40, 8256), (1100, 4160), (9, 16448)])
def test_in_place(T, d, dtype):
    g = torch.Generator().manual_seed(T + d)
    x, dres = (torch.randn(T, d, generator=g).cuda() for _ in range(2))
    y, du = (torch.randn(T, d, generator=g).to(dtype).cuda() for _ in range(2))
    gamma = (1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda()
    D = M.LayerDesc(d, 0, 0, 0, 0, 0, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32)
    want = M.mcft_residual_rmsnorm_mx8(D, x, y, gamma)
    stream, res = x.clone(), y.clone()
    got = M.mcft_residual_rmsnorm_mx8(D, stream, res, gamma, out=stream, u=res)
    M.mcft_device_error()
    assert got[0] is stream and got[1] is res and all(torch.equal(a, b) for a, b in zip(got, want))
    rstd, out = want[3], want[0]
    dx, dgamma = M.mcft_rmsnorm_grad(D, gamma, rstd, du, dres, x=out)
    for name in ("dres", "x") + (("du",) if dtype == F32 else ()):
        t = dict(dres=dres.clone(), x=out.clone(), du=du.clone())
        got = M.mcft_rmsnorm_grad(D, gamma, rstd, t["du"], t["dres"], x=t["x"], dx=t[name])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgamma), name
    M.mcft_device_error()
