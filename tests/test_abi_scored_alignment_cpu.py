"""Scored routing and the mx4 layer refuse 4-byte arrays that do not begin on 4 bytes, before a launch. No GPU."""
import ctypes as C

import pytest

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

P = C.c_void_p(4096)


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return M.lib()


@pytest.mark.parametrize("off", [1, 2, 3])
def test_refusals(off):
    L, bad = M.lib(), C.c_void_p(4096 + off)
    desc = M.ScoredDesc(128, 64, 4, 1, 1, 1, 0, 0, M.MCFT_BF16, 1.0)
    for at in (4, 5, 6, 7, 8):  # bias, idx, gate, logits, load
        a = [C.byref(desc), P, 4, P, P, P, P, P, P, None]
        a[at] = bad
        assert L.mcft_route_scored(*a) == M.MCFT_ERR_INVALID and b"misaligned" in L.mcft_last_error(), at
    need = M.mcft_route_scored_grad_workspace_size(desc, 4)
    for at in (4, 5, 6, 7):  # idx, gate, logits, dgate
        a = [C.byref(desc), P, 4, P, P, P, P, P, P, P, 0, P, need, None]
        a[at] = bad
        assert L.mcft_route_scored_grad(*a) == M.MCFT_ERR_INVALID and b"misaligned" in L.mcft_last_error(), at
    layer = M.LayerDesc(256, 8, 2, 512, 0, 0, M.MCFT_BF16)
    need = M.mcft_mx4_workspace_size(layer, 4)
    table = (C.c_void_p * 8)(*[4096] * 8)
    for at in (3, 4):  # idx, gate
        a = [C.byref(layer), P, 4, P, P, table, None, P, P, need, None]
        a[at] = bad
        assert L.mcft_moe_forward_mx4(*a) == M.MCFT_ERR_INVALID and b"misaligned" in L.mcft_last_error(), at
