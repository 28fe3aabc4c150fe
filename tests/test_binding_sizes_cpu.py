"""The Python binding of scored routing and of the mx4 operators refuses tensors that are smaller than the sizes that it is given, or of
another type or shape, before the library sees their addresses. No GPU: nothing is launched."""
import pytest
import torch

from paper_2609_34077_gb300 import build
from paper_2609_34077_gb300 import mcft as M

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    M.lib()


@pytest.fixture(autouse=True)
def no_launch(monkeypatch):
    """Every call that would launch says so instead."""
    class Library:
        def __getattr__(self, name):
            def call(*_):
                raise AssertionError(f"{name} was called")
            return call if name in ("mcft_route_scored", "mcft_route_scored_grad", "mcft_mx4_quantize", "mcft_mx4_dequantize",
                                    "mcft_mx4_matmul", "mcft_mx4_pack_expert", "mcft_moe_forward_mx4") else getattr(real, name)
    real = M.lib()
    monkeypatch.setattr(M, "lib", lambda: Library())
    monkeypatch.setattr(M, "_stream", lambda s: None)


def refused(call, good, **change):
    with pytest.raises(M.MCFTError) as e:
        call(**{**good, **change})
    assert e.value.status == M.MCFT_ERR_INVALID, change


def accepted(call, good, **change):
    with pytest.raises(AssertionError, match="was called"):
        call(**{**good, **change})


def mx4(rows, cols, less=0):
    return torch.zeros(M.mcft_mx4_size(rows, cols) - less, dtype=torch.uint8)


def test_quantise_and_back():
    for R, C in ((1, 1), (8, 128), (9, 129), (130, 300)):
        x = torch.zeros(R, C)
        accepted(M.mcft_mx4_quantize, dict(x=x, q=mx4(R, C)))
        refused(M.mcft_mx4_quantize, dict(x=x), q=mx4(R, C, 1))
        good = dict(q=mx4(R, C), rows=R, cols=C)
        accepted(M.mcft_mx4_dequantize, good, y=torch.zeros(R, C, dtype=BF16))
        for change in (dict(q=mx4(R, C, 1)), dict(rows=R + 128), dict(cols=C + 128), dict(y=torch.zeros(R, C + 1)), dict(y=torch.zeros(R + 1, C))):
            refused(M.mcft_mx4_dequantize, good, **change)


def test_product():
    good = dict(a=mx4(3, 300), b=mx4(200, 300), M=3, N=200, K=300)
    accepted(M.mcft_mx4_matmul, good)
    accepted(M.mcft_mx4_matmul, good, a=mx4(3, 1000), y=torch.zeros(3, 200))
    for change in (dict(a=mx4(3, 300, 1)), dict(b=mx4(200, 300, 1)), dict(M=200), dict(N=300), dict(K=385), dict(y=torch.zeros(200, 3)),
                   dict(y=torch.zeros(3, 199)), dict(y=torch.zeros(3, 201))):
        refused(M.mcft_mx4_matmul, good, **change)


def test_expert_blocks():
    desc = M.LayerDesc(128, 4, 2, 64, 0, 0, M.MCFT_BF16)
    good = dict(desc=desc, block=torch.zeros(3 * 64 * 128, dtype=BF16), out=torch.zeros(M.mcft_mx4_expert_size(desc), dtype=torch.uint8))
    accepted(M.mcft_mx4_pack_expert, good)
    for change in (dict(block=torch.zeros(3 * 64 * 128 - 1, dtype=BF16)), dict(block=torch.zeros(3 * 64 * 128)), dict(out=good["out"][:-1])):
        refused(M.mcft_mx4_pack_expert, good, **change)


def test_layer():
    desc = M.LayerDesc(128, 4, 2, 64, 0, 0, M.MCFT_BF16)
    good = dict(desc=desc, x=torch.zeros(5, 128, dtype=BF16), idx=torch.zeros(5, 2, dtype=I32), gate=torch.zeros(5, 2), experts=[4096] * 4)
    accepted(M.mcft_moe_forward_mx4, good)
    for change in (dict(x=torch.zeros(5, 128)), dict(x=torch.zeros(5, 64, dtype=BF16)), dict(idx=torch.zeros(5, 2, dtype=torch.int64)),
                   dict(idx=torch.zeros(4, 2, dtype=I32)), dict(gate=torch.zeros(5, 1)), dict(gate=torch.zeros(5, 2, dtype=BF16)),
                   dict(y=torch.zeros(4, 128, dtype=BF16)), dict(y=torch.zeros(5, 128))):
        refused(M.mcft_moe_forward_mx4, good, **change)


def test_routing():
    desc = M.ScoredDesc(128, 16, 2, 1, 1, 1, 0, 0, M.MCFT_F32, 1.0)
    good = dict(desc=desc, x=torch.zeros(5, 128), w_router=torch.zeros(16, 128), bias=torch.zeros(16), idx=torch.zeros(5, 2, dtype=I32),
                gate=torch.zeros(5, 2), logits=torch.zeros(5, 16), load=torch.zeros(16, dtype=I32))
    accepted(M.mcft_route_scored, good)
    accepted(M.mcft_route_scored, good, bias=None, idx=None, gate=None, logits=None, load=None)
    common = (dict(x=torch.zeros(5, 64)), dict(x=torch.zeros(5, 128, dtype=BF16)), dict(w_router=torch.zeros(15, 128)),
              dict(w_router=torch.zeros(16, 128, dtype=BF16)), dict(idx=torch.zeros(5, 2, dtype=torch.int64)),
              dict(idx=torch.zeros(4, 2, dtype=I32)), dict(gate=torch.zeros(5, 3)), dict(gate=torch.zeros(5, 2, dtype=torch.float64)),
              dict(logits=torch.zeros(5, 15)), dict(logits=torch.zeros(5, 16, dtype=BF16)))
    for change in common + (dict(bias=torch.zeros(15)), dict(bias=torch.zeros(16, dtype=BF16)), dict(load=torch.zeros(15, dtype=I32)),
                            dict(load=torch.zeros(16, dtype=torch.int64))):
        refused(M.mcft_route_scored, good, **change)
    good = {k: v for k, v in good.items() if k not in ("bias", "load")}
    good.update(dgate=torch.zeros(5, 2), dx=torch.zeros(5, 128), dw=torch.zeros(16, 128))
    accepted(M.mcft_route_scored_grad, good)
    for change in common + (dict(dgate=torch.zeros(5, 3)), dict(dx=torch.zeros(4, 128)), dict(dx=torch.zeros(5, 128, dtype=BF16)),
                            dict(dw=torch.zeros(16, 64)), dict(dw=torch.zeros(16, 128, dtype=BF16)), dict(dw=None, accumulate=True)):
        refused(M.mcft_route_scored_grad, good, **change)
