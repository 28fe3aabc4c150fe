"""Outputs at the address of an input or of another output, which would be written while they are read: refused on the host."""
import ctypes as C

import pytest

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

BAD = M.MCFT_ERR_INVALID
SIZE = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return M.lib()


def refused(st):
    text = M.lib().mcft_last_error()
    return st == BAD and (b"may not be" in text or b"are the same" in text)


def tensors(names):
    return {n: C.c_void_p((i + 1) << 20) for i, n in enumerate(names)}


def desc(dtype):
    return C.byref(M.LayerDesc(128, 0, 0, 192, 0, 0, dtype))


@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
def test_of_the_forward(dtype):
    for T in (3, 300):
        for a, b in (("y", "x"), ("y", "block"), ("y", "ckpt"), ("ckpt", "x"), ("ckpt", "block")):
            t = tensors(("x", "block", "y", "ckpt", "ws"))
            t[a] = t[b]
            assert refused(M.lib().mcft_ffn_forward(desc(dtype), t["x"], T, t["block"], t["y"], t["ckpt"], t["ws"], SIZE, None)), (a, b)


@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
def test_of_the_norm(dtype):
    ins, outs = ("x", "y", "gamma"), ("out", "u", "u8", "x8", "rstd")
    pairs = [(o, i) for o in outs for i in ins if (o, i) not in (("out", "x"), ("u", "y"))]
    pairs += [(a, b) for i, a in enumerate(outs) for b in outs[:i]]
    for a, b in pairs:
        t = tensors(ins + outs)
        t[a] = t[b]
        assert refused(M.lib().mcft_residual_rmsnorm_mx8(desc(dtype), t["x"], t["y"], 3, t["gamma"], C.c_float(1e-5), t["out"], t["u"],
                                                         t["u8"], t["x8"], t["rstd"], None)), (a, b)


@pytest.mark.parametrize("dtype", [M.MCFT_F32, M.MCFT_BF16])
def test_of_its_gradient(dtype):
    for form in ("x", "x8"):
        ins = (form, "rstd", "gamma", "du", "dres")
        allowed = {("dx", "dres"), ("dx", "x")} | ({("dx", "du")} if dtype == M.MCFT_F32 else set())
        for a, b in [(o, i) for o in ("dx", "dgamma") for i in ins if (o, i) not in allowed] + [("dx", "dgamma")]:
            t = tensors(ins + ("dx", "dgamma", "ws"))
            t[a] = t[b]
            assert refused(M.lib().mcft_rmsnorm_grad(desc(dtype), t.get("x"), t.get("x8"), t["rstd"], t["gamma"], t["du"], 3, t["dres"],
                                                     t["dx"], t["dgamma"], 0, t["ws"], SIZE, None)), (a, b)


def test_of_mx8():
    P = C.c_void_p(4096)
    assert refused(M.lib().mcft_mx8_quantize(P, 4, 32, 32, M.MCFT_BF16, P, None))
    assert refused(M.lib().mcft_mx8_dequantize(P, 4, 32, M.MCFT_F32, P, 32, None))
