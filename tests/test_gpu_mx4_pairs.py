"""mx4 products at the sizes that CTA pairs and few wide tiles take: odd numbers of token tiles, a last weight tile whose
second half is empty, an odd last stage, outputs of any width and stride. Bounds as in test_gpu_mx4."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M
from .test_gpu_mx4 import check_product, matrix, values
from .test_gpu_mx4_moe import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M_,N,K", [
    (1300, 3590, 2144),  # eleven token tiles, six rows in the last weight tile, seventeen chunks of the contraction
    (1537, 3840, 2048), (1409, 3713, 2049),
    (256, 5000, 300), (129, 4865, 1000), (640, 1999, 96)])  # single CTAs, fewer items than SMs
def test_product(M_, N, K, dtype):
    a, b = matrix(M_ + K, M_, K), matrix(N + K + 1, N, K, std=0.02)
    y = M.mcft_mx4_matmul(M.mcft_mx4_quantize(a.cuda()), M.mcft_mx4_quantize(b.cuda()), M_, N, K, dtype)
    M.mcft_device_error()
    check_product(y, values(a), values(b), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M_,N,K,ld,at", [(1290, 3591, 2080, 3600, 3), (300, 5121, 100, 5121, 0), (260, 4992, 64, 5003, 5)])
def test_nothing_beside_the_result_is_written(M_, N, K, ld, at, dtype):
    a, b = matrix(7, M_, K), matrix(8, N, K, std=0.02)
    out = torch.full((M_ + 2, ld), 9.0, dtype=dtype, device="cuda")
    M.mcft_mx4_matmul(M.mcft_mx4_quantize(a.cuda()), M.mcft_mx4_quantize(b.cuda()), M_, N, K, y=out[1:-1, at:at + N])
    M.mcft_device_error()
    check_product(out[1:-1, at:at + N], values(a), values(b), dtype)
    out[1:-1, at:at + N] = 9.0
    assert (out == 9).all()


def test_a_nan_block_stays_in_its_row_and_column():
    M_, N, K = 2000, 2600, 2112
    a, b = matrix(5, M_, K), matrix(6, N, K)
    a[M_ // 2, 40] = float("inf")
    b[N // 3, K - 1] = float("nan")
    y = M.mcft_mx4_matmul(M.mcft_mx4_quantize(a.cuda()), M.mcft_mx4_quantize(b.cuda()), M_, N, K, torch.float32).cpu()
    want = torch.zeros(M_, N, dtype=torch.bool)
    want[M_ // 2] = True
    want[:, N // 3] = True
    assert torch.equal(torch.isnan(y), want)


def test_a_layer_by_pairs_gives_the_bits_of_single_tiles():
    # 1500 tokens on two experts go by pairs, 300 by single tiles of the same width: the sums are the same (not in bf16,
    # where the larger call keeps the experts' outputs in 16 bits and the smaller in 32)
    L = Layer(2048, 2, 1, 2560, 1, torch.float32)
    x, idx, gate = L.batch(1500, drop=0.1)
    y = L.run(x, idx, gate)
    for at in (0, 300, 1200):
        part = slice(at, at + 300)
        assert torch.equal(y[part], L.run(x[part], idx[part], gate[part]))


def test_experts_with_odd_and_no_tiles_by_pairs():
    # tokens of the experts: none, one, 128, 129, 1100 and the rest; again by single tiles, 900 tokens at a time
    L = Layer(2048, 6, 1, 1024, 0, torch.float32)
    x, idx, gate = L.batch(3500)
    idx[:] = 5
    at = 0
    for e, n in enumerate([0, 1, 128, 129, 1100]):
        idx[at:at + n] = e
        at += n
    order = torch.randperm(len(x), generator=torch.Generator().manual_seed(3))
    idx = idx[order]
    y = L.run(x, idx, gate)
    for at in (0, 900, 1800, 2600):
        part = slice(at, at + 900)
        assert torch.equal(y[part], L.run(x[part], idx[part], gate[part]))
