"""Host-side argument checks and sizes of the mx4 operators and of scored routing, which need no GPU."""
import ctypes as C

import pytest

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

P = C.c_void_p(4096)


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return M.lib()


def test_sizes():
    assert M.mcft_mx4_size(0, 1) == 0
    assert M.mcft_mx4_size(1, 1) == 512 + 512  # one 8-row group of codes, one 128-row block of scales
    assert M.mcft_mx4_size(128, 128) == 128 * 64 + 512
    assert M.mcft_mx4_size(28672, 4096) == 28672 * 4096 * 17 // 32
    desc = M.LayerDesc(4096, 8, 2, 14336, 0, 0, M.MCFT_BF16)
    assert M.mcft_mx4_expert_size(desc) == 3 * 4096 * 14336 * 17 // 32


@pytest.mark.parametrize("shape", [(256, 8, 2, 512, 0), (2048, 64, 6, 1408, 2), (64, 1, 1, 64, 8), (128, 256, 16, 64, 0)])
@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
def test_a_workspace_serves_any_fewer_tokens(shape, dtype):
    d, E, K, w, S = shape
    desc = M.LayerDesc(d, E, K, w, S, 0, dtype)
    sizes = [M.mcft_mx4_workspace_size(desc, T) for T in [0, 1, 2, 3, 15, 16, 17, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257, 1000, 4096]]
    assert sizes == sorted(sizes) and sizes[0] == 0
    scored = M.ScoredDesc(d, E, min(K, E), 1, 1, 1, 0, 0, dtype, 1.0)
    sizes = [M.mcft_route_scored_grad_workspace_size(scored, T) for T in list(range(0, 700)) + [1000, 1999, 2000, 4096, 8192, 8200]]
    assert sizes == sorted(sizes) and sizes[0] == 0


def test_refusals_of_matrices():
    L = M.lib()
    n = C.c_size_t(0)
    assert L.mcft_mx4_size(-1, 4, C.byref(n)) == M.MCFT_ERR_INVALID
    assert L.mcft_mx4_size(4, 0, C.byref(n)) == M.MCFT_ERR_INVALID
    assert L.mcft_mx4_size(4, 4, None) == M.MCFT_ERR_INVALID
    for call in (lambda *a: L.mcft_mx4_quantize(a[0], *a[1:4], a[4], a[5], None),
                 lambda *a: L.mcft_mx4_dequantize(a[5], a[1], a[2], a[4], a[0], a[3], None)):
        assert call(P, -1, 4, 4, 1, P) == M.MCFT_ERR_INVALID
        assert call(P, 4, 0, 4, 1, P) == M.MCFT_ERR_INVALID
        assert call(P, 4, 64, 63, 1, P) == M.MCFT_ERR_INVALID
        assert b"stride" in L.mcft_last_error()
        assert call(P, 4, 64, 64, 2, P) == M.MCFT_ERR_INVALID
        assert call(None, 4, 64, 64, 1, P) == M.MCFT_ERR_INVALID
        assert call(P, 4, 64, 64, 1, None) == M.MCFT_ERR_INVALID
        assert call(P, 4, 64, 64, 1, C.c_void_p(4104)) == M.MCFT_ERR_INVALID
        assert call(C.c_void_p(4097), 4, 64, 64, 1, P) == M.MCFT_ERR_INVALID
        assert call(P, 2 ** 31, 64, 64, 1, P) == M.MCFT_ERR_UNSUPPORTED
        assert call(None, 0, 64, 64, 1, None) == M.MCFT_OK
    ok = [P, P, 4, 8, 64, 1, P, 8, None]
    for at, bad, status in ((0, None, 1), (1, None, 1), (2, -1, 1), (3, -1, 1), (4, 0, 1), (5, 3, 1), (6, None, 1), (7, 7, 1),
                            (0, C.c_void_p(4100), 1), (6, C.c_void_p(4097), 1)):
        a = list(ok)
        a[at] = bad
        assert L.mcft_mx4_matmul(*a) == status, (at, bad)
    a = list(ok)
    a[2], a[3], a[7] = 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31
    assert L.mcft_mx4_matmul(*a) == M.MCFT_ERR_UNSUPPORTED
    a = list(ok)
    a[2] = 0
    assert L.mcft_mx4_matmul(*a) == M.MCFT_OK


def test_refusals_of_layers():
    L = M.lib()
    desc = M.LayerDesc(256, 8, 2, 512, 1, 0, M.MCFT_BF16)
    table = (C.c_void_p * 8)(*[4096] * 8)
    shared = (C.c_void_p * 1)(4096)
    need = M.mcft_mx4_workspace_size(desc, 4)
    ok = [C.byref(desc), P, 4, P, P, table, shared, P, P, need, None]
    for at, bad in ((0, None), (1, None), (2, -1), (3, None), (4, None), (5, None), (6, None), (7, None), (8, None), (9, need - 1),
                    (1, C.c_void_p(4104)), (7, C.c_void_p(4104)), (8, C.c_void_p(4096 + 128)),
                    (5, (C.c_void_p * 8)(*[4100] * 8)), (6, (C.c_void_p * 1)(None))):
        a = list(ok)
        a[at] = bad
        assert L.mcft_moe_forward_mx4(*a) == M.MCFT_ERR_INVALID, at
        assert L.mcft_last_error()
    a = list(ok)
    a[2] = 0
    assert L.mcft_moe_forward_mx4(*a) == M.MCFT_OK
    assert L.mcft_mx4_pack_expert(C.byref(desc), None, P, None) == M.MCFT_ERR_INVALID
    assert L.mcft_mx4_pack_expert(C.byref(desc), P, C.c_void_p(4104), None) == M.MCFT_ERR_INVALID
    n = C.c_size_t(0)
    assert L.mcft_mx4_workspace_size(C.byref(desc), 2 ** 31 - 1, C.byref(n)) == M.MCFT_ERR_UNSUPPORTED


def test_refusals_of_routing():
    L = M.lib()
    good = dict(d=128, E=64, K=4, n_group=8, topk_group=2, group_top=1, score=0, gate=0, dtype=1, scale=1.0)
    n = C.c_size_t(0)
    for change, status in ((dict(d=100), 1), (dict(E=0), 1), (dict(E=264), 5), (dict(K=17), 5), (dict(n_group=7), 1), (dict(n_group=64), 5),
                           (dict(topk_group=0), 1), (dict(group_top=9), 1), (dict(group_top=3), 5), (dict(score=2), 1), (dict(scale=-1.0), 1)):
        desc = M.ScoredDesc(**{**good, **change})
        assert L.mcft_route_scored_grad_workspace_size(C.byref(desc), 4, C.byref(n)) == status, change
        assert L.mcft_route_scored(C.byref(desc), P, 4, P, None, P, P, None, None, None) == status
    desc = M.ScoredDesc(**good)
    for at in (1, 3, 5, 6):
        a = [C.byref(desc), P, 4, P, None, P, P, None, None, None]
        a[at] = None
        assert L.mcft_route_scored(*a) == M.MCFT_ERR_INVALID
    need = M.mcft_route_scored_grad_workspace_size(desc, 4)
    ok = [C.byref(desc), P, 4, P, P, P, P, P, P, P, 0, P, need, None]
    for at, bad in ((1, None), (3, None), (4, None), (5, None), (6, None), (7, None), (11, None), (12, need - 1), (2, -1),
                    (8, C.c_void_p(4104)), (9, C.c_void_p(4104)), (11, C.c_void_p(4096 + 128))):
        a = list(ok)
        a[at] = bad
        assert L.mcft_route_scored_grad(*a) == M.MCFT_ERR_INVALID, at
    a = list(ok)
    a[8] = a[9] = None
    assert L.mcft_route_scored_grad(*a) == M.MCFT_ERR_INVALID
