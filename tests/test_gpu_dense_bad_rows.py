"""What becomes of a token with an infinity in its input, or in its incoming gradient: none of its outputs is finite (no weight is zero), its
checkpoint's blocks read back as NaN, and other tokens' rows keep their bits. At token counts of every path: few tokens, fp32 weights
cut as they are read, products."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M
from tests.dense_model import Case

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [2, 9, 20, 40, 70, 300])
def test_an_infinite_token(T, dtype, value):
    c = Case(T, 192, 320, dtype)
    assert bool((c.block != 0).all())
    D = M.LayerDesc(192, 0, 0, 320, 0, 0, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32)
    ckpt = torch.empty(M.mcft_mx8_size(T, 640), dtype=torch.uint8, device="cuda")

    def step(x, dy):
        y = M.mcft_ffn_forward(D, x, c.block)
        z = M.mcft_ffn_forward(D, x, c.block, ckpt=ckpt)
        return (y, z, M.mcft_mx8_dequantize(ckpt, T, 640, F32), M.mcft_ffn_grad(D, dy, c.block, x=x)[0],
                M.mcft_ffn_grad(D, dy, c.block, x=x, ckpt=ckpt)[0])

    want = step(c.x, c.dy)
    rest = [t for t in range(T) if t != 1]
    x = c.x.clone()
    x[1, 3] = value
    got = step(x, c.dy)
    for a, b in zip(got, want):
        assert torch.equal(a[rest], b[rest])
        assert not bool(a[1].isfinite().any())
    assert bool(got[2][1].isnan().all())
    dy = c.dy.clone()
    dy[1, 5] = value
    got = step(c.x, dy)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
    for a, b in zip(got[3:], want[3:]):
        assert torch.equal(a[rest], b[rest])
        assert not bool(a[1].isfinite().any())
    M.mcft_device_error()
