"""mx4 quantisation and product against the fp64 oracle.

Rounding to the format is exact, so quantise + dequantise equals the oracle's values bit for bit. Products of
codes and scales are exact in fp32; a sum of n terms in fp32 (in any order, terms aligned to the largest of a
step) is within 2 n 2^-24 of the sum of the terms' magnitudes: the bound of the fp32 results, and with half a
unit of bf16 (2^-9 relative, 2^-8 allowed) of the bf16 ones."""
import numpy as np
import pytest
import torch

import oracle.mx4 as O
from paper_2609_34077_gb300 import mcft as M

pytestmark = pytest.mark.gpu


def matrix(seed, R, C, dtype=torch.bfloat16, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, C, generator=g) * std
    x[:, ::13] *= 16
    x[1::5] *= 2.0 ** -20
    return x.to(dtype)


def values(x):
    return O.quantize(x.double().numpy())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(1, 1), (1, 32), (3, 31), (7, 33), (8, 128), (9, 130), (129, 257), (64, 1024),
                                 (200, 1056), (5, 4100)])
def test_round_trip_is_exact(R, C, dtype):
    x = matrix(R * 1000 + C, R, C, dtype)
    q = M.mcft_mx4_quantize(x.cuda())
    assert q.numel() == M.mcft_mx4_size(R, C)
    ref = values(x)
    for out in (torch.float32, torch.bfloat16):
        y = M.mcft_mx4_dequantize(q, R, C, out)
        np.testing.assert_array_equal(y.cpu().double().numpy(), ref)


def test_every_tie_and_both_signs():
    a = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])
    x = torch.cat([a, -a]).reshape(1, 32) * 2.0 ** torch.arange(-100, 100, 7)[:, None]
    x = torch.cat([x, torch.nextafter(x, torch.tensor(9e37)), torch.nextafter(x, torch.tensor(-9e37))])
    y = M.mcft_mx4_dequantize(M.mcft_mx4_quantize(x.cuda()), *x.shape, torch.float32)
    np.testing.assert_array_equal(y.cpu().double().numpy(), values(x))


def test_zeros_extremes_and_non_finite_blocks():
    x = torch.zeros(9, 64)
    x[1, :32] = 2.0 ** -149  # subnormal: below half the smallest code
    x[2, :32] = 2.0 ** -126
    x[3] = 3.4028234e38
    x[4, 5], x[5, 40], x[6, 0] = float("inf"), float("nan"), float("-inf")
    x[7] = torch.linspace(-1e-37, 1e-37, 64)
    y = M.mcft_mx4_dequantize(M.mcft_mx4_quantize(x.cuda()), 9, 64, torch.float32)
    np.testing.assert_array_equal(y.cpu().double().numpy(), values(x))  # (NaN where the oracle has NaN)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_row_strides_and_offsets(dtype):
    base = matrix(3, 40, 301, dtype).cuda()
    for part in (base[:, 1:290], base[::3, 8:264], base[5:6, 3:4], base[2:30:2]):
        R, C = part.shape
        q = M.mcft_mx4_quantize(part)
        assert torch.equal(q, M.mcft_mx4_quantize(part.contiguous()))
        out = torch.full((R, C + 7), 5.0, dtype=dtype, device="cuda")
        M.mcft_mx4_dequantize(q, R, C, y=out[:, 3:3 + C])
        np.testing.assert_array_equal(out[:, 3:3 + C].cpu().double().numpy(), values(part.cpu()))
        assert (out[:, :3] == 5).all() and (out[:, 3 + C:] == 5).all()


def test_no_rows_and_refusals():
    x = torch.zeros(0, 32, device="cuda")
    assert M.mcft_mx4_quantize(x).numel() == 0
    assert M.mcft_mx4_dequantize(M.mcft_mx4_quantize(x), 0, 32).shape == (0, 32)
    q = torch.empty(4096, dtype=torch.uint8, device="cuda")
    one = torch.zeros(1, 32, device="cuda")
    with pytest.raises(M.MCFTError):
        M.mcft_mx4_quantize(one, q=q[1:])  # misaligned
    with pytest.raises(M.MCFTError):
        M.mcft_mx4_quantize(one.expand(4, 32), q=q)  # rows on top of each other
    with pytest.raises(KeyError):
        M.mcft_mx4_quantize(one.half())
    with pytest.raises(M.MCFTError):
        M.mcft_mx4_matmul(q, q, 1, 1, 0)
    with pytest.raises(M.MCFTError):
        M.mcft_mx4_matmul(q[4:], q, 1, 1, 32)
    assert M.mcft_mx4_matmul(q, q, 0, 5, 32).shape == (0, 5)


def check_product(y, a, b, dtype):
    ref = a @ b.T
    n = a.shape[1]
    tol = 2 * n * 2.0 ** -24 * (np.abs(a) @ np.abs(b).T)
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(ref)
    err = np.abs(y.cpu().double().numpy() - ref)
    assert (err <= tol + 1e-300).all(), f"worst {np.max(err / (tol + 1e-300)):.3g} of the bound"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M_,N,K", [
    (1, 1, 1), (1, 64, 64), (8, 64, 128), (5, 130, 192), (1, 4096, 4096), (17, 96, 2080), (128, 128, 256),
    (129, 65, 33), (300, 700, 1440), (64, 2048, 1408), (257, 513, 95), (1024, 4864, 512), (2500, 4000, 224)])
def test_product(M_, N, K, dtype):
    a, b = matrix(M_ + K, M_, K), matrix(N + K + 1, N, K, std=0.02)
    y = M.mcft_mx4_matmul(M.mcft_mx4_quantize(a.cuda()), M.mcft_mx4_quantize(b.cuda()), M_, N, K, dtype)
    M.mcft_device_error()
    check_product(y, values(a), values(b), dtype)


def test_product_into_a_strided_result_and_on_another_stream():
    a, b = matrix(1, 70, 320), matrix(2, 200, 320)
    out = torch.full((70, 233), 7.0, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        M.mcft_mx4_matmul(M.mcft_mx4_quantize(a.cuda()), M.mcft_mx4_quantize(b.cuda()), 70, 200, 320, y=out[:, 5:205])
    s.synchronize()
    check_product(out[:, 5:205], values(a), values(b), torch.float32)
    assert (out[:, :5] == 7).all() and (out[:, 205:] == 7).all()


@pytest.mark.parametrize("M_,N,K", [(3, 200, 320), (2000, 2600, 192)])
def test_a_nan_block_stays_in_its_row_and_column(M_, N, K):
    a, b = matrix(5, M_, K), matrix(6, N, K)
    a[M_ // 2, 40] = float("inf")
    b[N // 3, K - 1] = float("nan")
    y = M.mcft_mx4_matmul(M.mcft_mx4_quantize(a.cuda()), M.mcft_mx4_quantize(b.cuda()), M_, N, K, torch.float32).cpu()
    nan = torch.isnan(y)
    want = torch.zeros(M_, N, dtype=torch.bool)
    want[M_ // 2] = True
    want[:, N // 3] = True
    assert torch.equal(nan, want)
