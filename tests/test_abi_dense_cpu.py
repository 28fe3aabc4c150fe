"""Host-side argument checks and sizes of the dense block, its checkpoints and the norm, which need no GPU."""
import ctypes as C

import pytest
import torch

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

P = C.c_void_p(4096)
ODD = C.c_void_p(4104)
BAD, LARGE = M.MCFT_ERR_INVALID, M.MCFT_ERR_UNSUPPORTED
EPS = C.c_float(1e-5)


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return M.lib()


def desc(d=128, w=192, dtype=M.MCFT_BF16):
    return M.LayerDesc(d, 0, 0, w, 0, 0, dtype)  # (E, K, n_shared and gate are not read)


def test_mx8_sizes():
    assert M.mcft_mx8_size(0, 1) == 0
    assert M.mcft_mx8_size(1, 1) == 33 and M.mcft_mx8_size(3, 33) == 3 * 66
    assert M.mcft_mx8_size(4096, 28672) == 4096 * 28672 * 33 // 32
    n = C.c_size_t(0)
    for args, st in (((-1, 4), BAD), ((4, 0), BAD), ((1 << 31, 4), LARGE), ((4, 536862721), LARGE)):
        assert M.lib().mcft_mx8_size(*args, C.byref(n)) == st
    assert M.lib().mcft_mx8_size(4, 4, None) == BAD


def test_refusals_of_mx8():
    L = M.lib()
    for call in (lambda x, r, c, ld, t, q: L.mcft_mx8_quantize(x, r, c, ld, t, q, None),
                 lambda x, r, c, ld, t, q: L.mcft_mx8_dequantize(q, r, c, t, x, ld, None)):
        assert call(None, 4, 4, 4, 1, P) == BAD and call(P, 4, 4, 4, 1, None) == BAD
        assert call(P, -1, 4, 4, 1, P) == BAD and call(P, 4, 0, 4, 1, P) == BAD
        assert call(P, 4, 64, 63, 1, P) == BAD and call(P, 4, 64, 64, 2, P) == BAD
        assert call(C.c_void_p(4098), 4, 4, 4, 0, P) == BAD and call(C.c_void_p(4097), 4, 4, 4, 1, P) == BAD
        assert call(P, 4, 4, 4, 1, ODD) == BAD and call(P, 4, 4, (1 << 40) + 1, 1, P) == LARGE
        assert call(None, 0, 4, 4, 1, None) == M.MCFT_OK


@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
@pytest.mark.parametrize("d,w", [(64, 64), (64, 14336), (4096, 64), (2048, 1408), (960, 704)])
def test_a_workspace_serves_any_fewer_tokens(d, w, dtype):
    D = desc(d, w, dtype)
    T = list(range(0, 70)) + [127, 128, 129, 255, 256, 257, 1000, 4096, 32768]
    for size in (M.mcft_ffn_workspace_size, M.mcft_ffn_grad_workspace_size, M.mcft_rmsnorm_grad_workspace_size):
        sizes = [size(D, t) for t in T]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[1] > 0


def test_refusals_of_descs():
    n = C.c_size_t(0)
    for size in (M.lib().mcft_ffn_workspace_size, M.lib().mcft_ffn_grad_workspace_size, M.lib().mcft_rmsnorm_grad_workspace_size):
        assert size(None, 1, C.byref(n)) == BAD and size(C.byref(desc()), 1, None) == BAD
        assert size(C.byref(desc()), -1, C.byref(n)) == BAD
        assert size(C.byref(desc()), (1 << 24) + 1, C.byref(n)) == LARGE
        for bad in (desc(d=0), desc(d=100), desc(dtype=2)):
            assert size(C.byref(bad), 1, C.byref(n)) == BAD
        assert size(C.byref(desc(d=(1 << 20) + 64)), 1, C.byref(n)) == LARGE
    assert M.lib().mcft_ffn_workspace_size(C.byref(desc(w=100)), 1, C.byref(n)) == BAD
    assert M.lib().mcft_ffn_workspace_size(C.byref(desc(w=(1 << 20) + 64)), 1, C.byref(n)) == LARGE
    assert M.lib().mcft_rmsnorm_grad_workspace_size(C.byref(desc(d=32768 + 64)), 1, C.byref(n)) == LARGE


def test_refusals_of_the_norm():
    def call(D=desc(), x=P, y=P, T=3, gamma=P, eps=EPS, out=P, u=P, u8=P, x8=P, rstd=P):
        return M.lib().mcft_residual_rmsnorm_mx8(C.byref(D) if D else None, x, y, T, gamma, eps, out, u, u8, x8, rstd, None)

    assert call(D=None) == BAD and call(T=-1) == BAD and call(x=None) == BAD and call(gamma=None) == BAD
    assert call(eps=C.c_float(-1.0)) == BAD and call(eps=C.c_float(2.0)) == BAD and call(eps=C.c_float(float("nan"))) == BAD
    assert call(out=None, u=None, u8=None, x8=None, rstd=None) == BAD
    for name in ("x", "y", "gamma", "out", "u", "u8", "x8"):
        assert call(**{name: ODD}) == BAD
    assert call(rstd=C.c_void_p(4098)) == BAD and call(D=desc(d=65536)) == LARGE
    assert call(T=0, x=None, gamma=None) == M.MCFT_OK


def test_refusals_of_its_gradient():
    size = 1 << 30

    def call(D=desc(), x=P, x8=None, rstd=P, gamma=P, du=P, T=3, dres=P, dx=P, dgamma=P, ws=P, n=size):
        return M.lib().mcft_rmsnorm_grad(C.byref(D) if D else None, x, x8, rstd, gamma, du, T, dres, dx, dgamma, 0, ws, n, None)

    assert call(D=None) == BAD and call(T=-1) == BAD and call(dx=None, dgamma=None) == BAD
    assert call(x8=P) == BAD and call(x=None) == BAD
    for name in ("rstd", "gamma", "du", "ws"):
        assert call(**{name: None}) == BAD
    for name in ("x", "gamma", "du", "dres", "dx", "dgamma", "ws"):
        assert call(**{name: ODD}) == BAD
    assert call(x=None, x8=ODD) == BAD and call(n=4) == BAD


def test_refusals_of_the_block():
    size = 1 << 40

    def call(D=desc(), x=P, T=3, block=P, y=P, ckpt=P, ws=P, n=size):
        return M.lib().mcft_ffn_forward(C.byref(D) if D else None, x, T, block, y, ckpt, ws, n, None)

    assert call(D=None) == BAD and call(T=-1) == BAD and call(T=(1 << 24) + 1) == LARGE
    for name in ("x", "block", "y", "ws"):
        assert call(**{name: None}) == BAD
    for name in ("x", "block", "y", "ckpt", "ws"):
        assert call(**{name: ODD}) == BAD
    assert call(n=M.mcft_ffn_workspace_size(desc(), 3) - 1) == BAD
    assert call(T=0, x=None, block=None, y=None, ws=None) == M.MCFT_OK


def test_refusals_of_its_gradient_too():
    size = 1 << 40

    def call(D=desc(), dy=P, T=3, block=P, x=P, x8=None, ckpt=P, dx=P, dblock=P, gt=M.MCFT_BF16, ws=P, n=size):
        return M.lib().mcft_ffn_grad(C.byref(D) if D else None, dy, T, block, x, x8, ckpt, dx, dblock, gt, 0, ws, n, None)

    assert call(D=None) == BAD and call(T=-1) == BAD and call(dx=None, dblock=None) == BAD
    assert call(gt=2) == BAD and call(D=desc(dtype=M.MCFT_F32)) == BAD  # bf16 gradients of an fp32 block
    assert call(x8=P) == BAD and call(x=None) == BAD and call(x=None, ckpt=None, dblock=None) == BAD
    for name in ("dy", "block", "ws"):
        assert call(**{name: None}) == BAD
    for name in ("dy", "block", "x", "ckpt", "dx", "dblock", "ws"):
        assert call(**{name: ODD}) == BAD
    assert call(n=M.mcft_ffn_grad_workspace_size(desc(), 3) - 1) == BAD
    assert call(T=0, dy=None, block=None, x=None, ckpt=None, dblock=None, ws=None) == M.MCFT_OK


def test_outputs_at_an_inputs_address_are_refused():
    at = [C.c_void_p(1 << 20 | i << 12) for i in range(9)]
    n, D = 1 << 40, C.byref(desc())
    x, block, y, ckpt, ws = at[:5]
    assert M.lib().mcft_ffn_forward(D, x, 3, block, x, ckpt, ws, n, None) == BAD
    assert b"y may not be x" in M.lib().mcft_last_error()
    dx, dblock = at[5:7]
    for out in ((y, dblock), (dx, y), (x, dblock), (dx, x), (dx, block), (ckpt, dblock), (dx, dx)):
        assert M.lib().mcft_ffn_grad(D, y, 3, block, x, None, ckpt, *out, M.MCFT_BF16, 0, ws, n, None) == BAD
        assert b"may not be inputs" in M.lib().mcft_last_error() or b"are the same" in M.lib().mcft_last_error()
    assert M.lib().mcft_ffn_grad(D, y, 3, block, None, x, ckpt, x, None, M.MCFT_BF16, 0, ws, n, None) == BAD


def test_the_binding_refuses_tensors_of_other_sizes():
    D, b, f = desc(), torch.bfloat16, torch.float32
    x, block, g = torch.zeros(5, 128, dtype=b), torch.zeros(3 * 128 * 192, dtype=b), torch.zeros(128, dtype=b)
    xs, n8, n8w = torch.zeros(5, 128), M.mcft_mx8_size(5, 128), M.mcft_mx8_size(5, 384)
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    calls = [
        lambda: M.mcft_mx8_quantize(xs, q=u8(n8 - 1)),
        lambda: M.mcft_mx8_dequantize(u8(n8 - 1), 5, 128),
        lambda: M.mcft_mx8_dequantize(u8(n8), 5, 128, y=torch.zeros(4, 128)),
        lambda: M.mcft_ffn_forward(D, x.float(), block),
        lambda: M.mcft_ffn_forward(D, x[:, :64].contiguous(), block),
        lambda: M.mcft_ffn_forward(D, x, block[1:]),
        lambda: M.mcft_ffn_forward(D, x, block, y=x[:4]),
        lambda: M.mcft_ffn_forward(D, x, block, ckpt=u8(n8w - 1)),
        lambda: M.mcft_ffn_grad(D, x, block),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, x8=u8(n8)),
        lambda: M.mcft_ffn_grad(D, x, block, x=x[:4]),
        lambda: M.mcft_ffn_grad(D, x, block, x8=u8(n8 - 1)),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, ckpt=u8(n8w - 1)),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, dx=x[:4]),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, accumulate=True),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, dblock=block[1:]),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, dblock=block.to(torch.float16)),
        lambda: M.mcft_ffn_grad(D, x, block, x=x, dblock=block, grad_dtype=f),
        lambda: M.mcft_residual_rmsnorm_mx8(D, x, None, g),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, xs, g),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, None),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, g[:64]),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, g, out=xs[:4]),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, g, u=xs),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, g, u8=u8(n8 - 1)),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, g, x8=u8(n8 - 1)),
        lambda: M.mcft_residual_rmsnorm_mx8(D, xs, x, g, rstd=torch.zeros(4)),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x, x=xs, x8=u8(n8)),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(4), x, x=xs),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), xs, x=xs),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x, x8=u8(n8 - 1)),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x, x=xs, dres=x),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x, x=xs, dx=xs[:4]),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x, x=xs, accumulate=True),
        lambda: M.mcft_rmsnorm_grad(D, g, torch.zeros(5), x, x=xs, dgamma=torch.zeros(64)),
    ]
    for i, c in enumerate(calls):
        with pytest.raises(M.MCFTError) as e:
            c()
        assert e.value.status == BAD, i
