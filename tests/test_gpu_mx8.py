"""mx8 quantisation and its inverse against the oracle, bit for bit: odd sizes, strides and alignments, the ends of the
exponents' range, NaN and infinities, guard regions, and a matrix whose offsets pass 32 bits."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_34077_gb300 import mcft as M
from tests.test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def parts(q, R, C):
    cp = -(-C // 32) * 32
    q = q.cpu().numpy()
    return q[: R * cp].reshape(R, cp), q[R * cp: R * cp // 32 * 33].reshape(R, cp // 32)


def values(R, C, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, C, generator=g) * torch.exp2(torch.randint(-12, 12, (R, 1), generator=g).float())
    x[:, ::17] *= 50
    return x.to(dtype)


def check(x, q, R, C):
    want, codes, scales = oracle.dense.mx8(x.double().cpu().numpy())
    got_codes, got_scales = parts(q, R, C)
    assert np.array_equal(got_scales, scales)
    ok = np.repeat(scales != 255, 32, 1)
    assert np.array_equal(got_codes[ok], codes[ok])
    return want


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,C", [(1, 1), (1, 31), (3, 33), (16, 64), (5, 96), (7, 1000), (130, 5295), (33, 8192), (2, 20000)])
def test_there_and_back(R, C, dtype):
    x = values(R, C, R * C, dtype).cuda()
    guard = Guarded(M.mcft_mx8_size(R, C)), Guarded(R * C * x.element_size())
    q = M.mcft_mx8_quantize(x, q=guard[0].view())
    want = check(x, q, R, C)
    y = M.mcft_mx8_dequantize(q, R, C, y=guard[1].view(dtype, (R, C)))
    assert np.array_equal(y.double().cpu().numpy(), want)
    for g in guard:
        g.check(f"{R} x {C}")
    M.mcft_device_error()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off,ld", [(0, 256), (1, 257), (8, 264), (3, 200), (16, 208)])
def test_strides(off, ld, dtype):
    R, C = 37, 190
    base = values(1, off + R * ld, 5, dtype).flatten().cuda()
    x = base.as_strided((R, C), (ld, 1), off)
    q = M.mcft_mx8_quantize(x)
    want = check(x, q, R, C)
    out = torch.full_like(base, 7.0)
    y = out.as_strided((R, C), (ld, 1), off)
    M.mcft_mx8_dequantize(q, R, C, y=y)
    assert np.array_equal(y.double().cpu().numpy(), want)
    y.fill_(7.0)
    assert bool((out == 7.0).all())  # nothing between the rows


@pytest.mark.parametrize("shift", [0, 1])
def test_ends_of_the_range(shift):
    big = [3.3e38, 448.0, 449.0, 464.0, 1.75, np.nextafter(np.float32(1.75), np.float32(2)), 1e-38, 1e-40, 1.4e-45, 448 * 2.0 ** -127, 0.0, -0.0]
    x = torch.zeros(len(big), 64 + shift)
    for i, b in enumerate(big):
        x[i, :32] = torch.tensor(np.float32(b)) * torch.linspace(-1, 1, 32)
        x[i, 31 if i % 2 else 0] = float(np.float32(b))
    x[3, 40], x[5, 63], x[6, 33] = float("nan"), float("inf"), float("-inf")
    x = x.cuda()
    q = M.mcft_mx8_quantize(x)
    want = check(x, q, *x.shape)
    got = M.mcft_mx8_dequantize(q, *x.shape, F32).double().cpu().numpy()
    assert np.array_equal(got, want, equal_nan=True)
    near = M.mcft_mx8_dequantize(q, *x.shape, BF16).float().cpu()
    assert torch.equal(torch.nan_to_num(near), torch.nan_to_num(torch.from_numpy(want).float().bfloat16().float()))


def test_no_rows():
    x = torch.empty(0, 40, device="cuda")
    assert M.mcft_mx8_dequantize(M.mcft_mx8_quantize(x), 0, 40).shape == (0, 40)


def test_offsets_past_32_bits():
    R, C = 66_000, 65_600  # 4.3e9 values
    x = torch.empty(R, C, dtype=BF16, device="cuda").fill_(0.75)
    x[-3:] = values(3, C, 9, BF16).cuda()
    q = M.mcft_mx8_quantize(x)
    want, codes, scales = oracle.dense.mx8(x[-3:].double().cpu().numpy())
    n = R * C
    assert np.array_equal(q[n - 3 * C: n].cpu().numpy().reshape(3, C), codes)
    assert np.array_equal(q[n + n // 32 - 3 * C // 32: n + n // 32].cpu().numpy().reshape(3, -1), scales)
    x.fill_(1.0)
    M.mcft_mx8_dequantize(q, R, C, y=x)
    assert np.array_equal(x[-3:].double().cpu().numpy(), want) and bool((x[:4] == 0.75).all())
