"""The widest mx4 matrices: one column more is refused before a launch is tried, by every call alike. No GPU: the calls that pass the
checks have no rows."""
import ctypes as C

import pytest

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

P = C.c_void_p(4096)
WIDEST = 65535 * 2048  # (the launch's second extent times its step; mx4_quant.cu)


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return M.lib()


def size(rows, cols):
    n = C.c_size_t(0)
    return M.lib().mcft_mx4_size(rows, cols, C.byref(n)), n.value


def test_the_size_of_a_matrix():
    assert size(1, WIDEST) == (M.MCFT_OK, WIDEST // 128 * (512 + 512))
    for rows, cols in ((1, WIDEST + 1), (1, 2 ** 62), (2 ** 31 - 128, 1), (2 ** 62, 2 ** 62)):
        assert size(rows, cols)[0] == M.MCFT_ERR_UNSUPPORTED


def test_quantise_and_back():
    L = M.lib()
    assert L.mcft_mx4_quantize(P, 0, WIDEST, WIDEST, M.MCFT_BF16, P, None) == M.MCFT_OK
    assert L.mcft_mx4_dequantize(P, 0, WIDEST, M.MCFT_BF16, P, WIDEST, None) == M.MCFT_OK
    for cols in (WIDEST + 1, 2 ** 30 - 1, 2 ** 40):
        for rows in (0, 1):
            assert L.mcft_mx4_quantize(P, rows, cols, cols, M.MCFT_BF16, P, None) == M.MCFT_ERR_UNSUPPORTED
            assert L.mcft_mx4_dequantize(P, rows, cols, M.MCFT_BF16, P, cols, None) == M.MCFT_ERR_UNSUPPORTED


def test_product():
    L = M.lib()
    assert L.mcft_mx4_matmul(P, P, 0, 8, WIDEST, M.MCFT_BF16, P, 8, None) == M.MCFT_OK
    for K in (WIDEST + 1, 2 ** 31 - 1):  # (its 64-column steps would pass an int)
        assert L.mcft_mx4_matmul(P, P, 1, 8, K, M.MCFT_BF16, P, 8, None) == M.MCFT_ERR_UNSUPPORTED
