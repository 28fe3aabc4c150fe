"""Scored routing and its gradient on tensors that begin in the middle of larger buffers: the bits of tensors of their own, and
nothing beside them is written."""
import pytest
import torch

from paper_2609_34077_gb300 import mcft as M

from .test_gpu_route_scored import desc_of

pytestmark = pytest.mark.gpu


def inside(offset, dtype, *shape):
    """A contiguous tensor that begins `offset` elements into a buffer, and the buffer."""
    n = 1
    for s in shape:
        n *= s
    buf = torch.full((n + offset + 64,), 7.0, dtype=dtype, device="cuda")
    return buf[offset:offset + n].view(shape), buf


def untouched(buf, offset, n):
    return (buf[:offset] == 7).all() and (buf[offset + n:] == 7).all()


def inputs(T, d, E, dtype):
    g = torch.Generator().manual_seed(T + E)
    return (torch.randn(T, d, generator=g).to(dtype).cuda(), (torch.randn(E, d, generator=g) * 0.05).to(dtype).cuda())


# up to 64 tokens a cluster of CTAs for four of them, then fp32 tiles or the tensor cores; bf16 of 256 experts of width 2048 always those
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d,E,K", [(1, 256, 256, 8), (9, 128, 68, 4), (9, 2048, 256, 8), (70, 192, 256, 8), (300, 128, 100, 3), (40, 64, 64, 6)])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_logits_anywhere(T, d, E, K, dtype, offset):
    x, w = inputs(T, d, E, dtype)
    D = desc_of(d, E, K, dtype, "sigmoid")
    want = torch.empty(T, E, device="cuda")
    idx, gate = M.mcft_route_scored(D, x, w, logits=want)
    logits, buf = inside(offset, torch.float32, T, E)
    assert logits.data_ptr() % 16 == 4 * offset
    idx2, gate2 = M.mcft_route_scored(D, x, w, logits=logits)
    M.mcft_device_error()
    assert torch.equal(logits, want) and torch.equal(idx, idx2) and torch.equal(gate, gate2)
    assert untouched(buf, offset, T * E)
    dg = torch.randn(T, K, generator=torch.Generator().manual_seed(1)).cuda()
    a, b = (M.mcft_route_scored_grad(D, x, w, idx, gate, z, dg) for z in (want, logits))
    M.mcft_device_error()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# up to 64 tokens and fp32 by multiply-adds, else the tensor cores; 16-byte offsets of which one is on 32 bytes
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d,E,K", [(3, 256, 64, 4), (64, 128, 256, 8), (65, 64, 16, 2), (300, 320, 100, 3), (1100, 2048, 256, 8)])
@pytest.mark.parametrize("at", [16, 32, 48])
def test_gradients_on_16_bytes(T, d, E, K, dtype, at):
    x, w = inputs(T, d, E, dtype)
    D = desc_of(d, E, K, dtype, "sigmoid")
    logits = torch.empty(T, E, device="cuda")
    idx, gate = M.mcft_route_scored(D, x, w, logits=logits)
    dg = torch.randn(T, K, generator=torch.Generator().manual_seed(1)).cuda()
    want = M.mcft_route_scored_grad(D, x, w, idx, gate, logits, dg)
    dx, xbuf = inside(at // x.element_size(), dtype, T, d)
    dw, wbuf = inside(at // 4, torch.float32, E, d)
    assert dx.data_ptr() % 32 == at % 32 == dw.data_ptr() % 32
    M.mcft_route_scored_grad(D, x, w, idx, gate, logits, dg, dx=dx, dw=dw)
    M.mcft_device_error()
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    assert untouched(xbuf, at // x.element_size(), T * d) and untouched(wbuf, at // 4, E * d)


def test_a_dx_off_16_bytes_is_refused():
    x, w = inputs(70, 64, 16, torch.bfloat16)
    D = desc_of(64, 16, 2, torch.bfloat16)
    logits = torch.empty(70, 16, device="cuda")
    idx, gate = M.mcft_route_scored(D, x, w, logits=logits)
    for offset in (1, 4, 7):
        with pytest.raises(M.MCFTError) as e:
            M.mcft_route_scored_grad(D, x, w, idx, gate, logits, gate, dx=inside(offset, torch.bfloat16, 70, 64)[0])
        assert e.value.status == M.MCFT_ERR_INVALID
    M.mcft_device_error()
