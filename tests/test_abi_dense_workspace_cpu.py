"""Workspaces of the dense block: what a call of few tokens of an fp32 layer wants does not hold the block a second time, since its
kernels cut the weights as they read them (the forward up to 64 tokens, the gradient up to 32)."""
import ctypes as C

import pytest

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return M.lib()


def section(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("d,w", [(64, 64), (1024, 2816), (4096, 14336), (1 << 20, 1 << 20)])
def test_few_tokens_of_fp32_layers_hold_no_block(d, w):
    D = M.LayerDesc(d, 0, 0, w, 0, 0, M.MCFT_F32)
    for T in (1, 2, 31, 32, 33, 63, 64):
        parts = section(6 * T * d)
        want = section(6 * T * w) + section(8 * T * w) + parts  # h in parts, g and u, x in parts
        assert M.mcft_ffn_workspace_size(D, T) == want
        if T <= 32:  # x's values, h, dg and du in parts, g and u, dh, x and dy in parts
            want = section(4 * T * d) + section(6 * T * w) + section(12 * T * w) + section(8 * T * w) + section(4 * T * w) + 2 * parts
            assert M.mcft_ffn_grad_workspace_size(D, T) == want
    block = 18 * d * w
    assert M.mcft_ffn_workspace_size(D, 65) > block and M.mcft_ffn_grad_workspace_size(D, 33) > block


@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
def test_a_workspace_serves_every_smaller_call(dtype):
    for d, w in ((64, 64), (64, 8192), (8192, 64), (704, 960)):
        D = M.LayerDesc(d, 0, 0, w, 0, 0, dtype)
        for size in (M.mcft_ffn_workspace_size, M.mcft_ffn_grad_workspace_size):
            sizes = [size(D, t) for t in range(0, 300)]
            assert sizes == sorted(sizes)


def test_less_is_refused():
    n, P = C.c_size_t(0), C.c_void_p(1 << 20)
    at = [C.c_void_p((i + 2) << 20) for i in range(4)]
    D = M.LayerDesc(128, 0, 0, 192, 0, 0, M.MCFT_F32)
    for T in (1, 32, 64):
        assert M.lib().mcft_ffn_workspace_size(C.byref(D), T, C.byref(n)) == M.MCFT_OK
        assert M.lib().mcft_ffn_forward(C.byref(D), at[0], T, at[1], at[2], None, P, n.value - 1, None) == M.MCFT_ERR_INVALID
        assert b"needed" in M.lib().mcft_last_error()
